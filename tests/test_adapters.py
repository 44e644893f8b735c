"""muxq_adapters: Y = base + s * (X A^T) B^T with the adapter of every row's request, against the formula in 64 bits.

Tolerances.  Products of two fp16 values are exact in fp32.  A matrix instruction adds 16 of them to its fp32 accumulator; what it loses there is
at most a step of fp32, 2^-22 of the sum of magnitudes so far when the addends are cut off instead of rounded.  With at most K / 16 such steps
in a row and 16 partial sums, T is off by at most (K / 16 + 16) 2^-22 sum|x a|.  As two fp16 numbers T loses 2^-22 of its value (half a step of a half step),
and 2^-25 / 2^13 = 2^-38 of the largest of its row where the lower number is subnormal.  The second product has two instructions per 16 ranks:
(r / 8 + 4) 2^-22 sum|T b|.  Scale and sum with base are two roundings of fp32, 2^-24 each.  A result in fp16 is off by half a step more: 2^-11 of the value, 2^-25 where it
is subnormal."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

F16, F32 = torch.float16, torch.float32


@pytest.fixture(scope="module")
def mx():
    from paper_2604_04701_b200 import build
    build.build()
    import paper_2604_04701_b200 as m
    m.lib()
    return m


@pytest.fixture
def gpu(mx):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return mx


def reference(X, A, B, ids, scale, rank, base):
    """(Y, bound of its error before it is rounded) in 64 bits; ids that are no slots count as none"""
    X, A, B, ids = X.double().cpu(), A.cpu(), B.cpu(), ids.cpu()
    M, K, S, R, N = X.shape[0], X.shape[1], A.shape[0], A.shape[1], B.shape[1]
    Y = torch.zeros(M, N, dtype=torch.float64) if base is None else base.double().cpu()
    E = torch.zeros_like(Y)
    for a in range(S):
        r = R if rank is None else int(rank[a])
        rows = (ids == a).nonzero()[:, 0]
        if not 0 < r <= R or not len(rows):
            continue
        x, A1, B1 = X[rows], A[a, :r].double(), B[a, :, :r].double()
        s = 1.0 if scale is None else float(scale[a])
        T = x @ A1.T
        eT = (K / 16 + 16) * 2.0 ** -22 * (x.abs() @ A1.abs().T) + 2.0 ** -22 * T.abs() + 2.0 ** -38 * T.abs().amax(1, keepdim=True)
        d = s * (T @ B1.T)
        Y[rows] += d
        E[rows] = abs(s) * (eT @ B1.abs().T + (r / 8 + 4) * 2.0 ** -22 * (T.abs() @ B1.abs().T)) + 2 * 2.0 ** -24 * d.abs()
    return Y, E


def check(got, want, err):
    half = (lambda v: v * 2.0 ** -11 + 2.0 ** -25) if got.dtype == F16 else (lambda v: v * 2.0 ** -24)
    assert torch.isfinite(got).all()
    off, tol = (got.double().cpu() - want).abs(), err + half(want.abs() + err)
    assert (off <= tol).all(), float((off / tol.clamp(min=1e-300)).max())


# ------------------------------------------------------------------------------------------------ refusals, without a GPU
class _CSet(ctypes.Structure):
    _fields_ = [("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("lda", ctypes.c_int), ("ldb", ctypes.c_int), ("sa", ctypes.c_int64), ("sb", ctypes.c_int64),
                ("scale", ctypes.c_void_p), ("rank", ctypes.c_void_p), ("slots", ctypes.c_int), ("max_rank", ctypes.c_int)]


def _call(mx, **over):
    """A call that would be valid but for what `over` says; its pointers are never dereferenced, so everything here has to be refused."""
    v = dict(X=0x100000, M=4, K=64, ldx=64, A=0x200000, B=0x300000, lda=64, ldb=16, sa=1024, sb=2048, scale=0x410000, rank=0x420000, slots=3, R=16, ids=0x430000, N=128,
             base=0x500000, ldbase=128, Y=0x600000, ldy=128, kind=0, status=0x440000, set=True)
    v.update(over)
    p = lambda a: None if a is None else ctypes.c_void_p(a)
    s = _CSet(v["A"], v["B"], v["lda"], v["ldb"], v["sa"], v["sb"], v["scale"], v["rank"], v["slots"], v["R"])
    return mx.lib().muxq_adapters(p(v["X"]), v["M"], v["K"], v["ldx"], ctypes.byref(s) if v["set"] else None, p(v["ids"]), v["N"], p(v["base"]), v["ldbase"],
                                  p(v["Y"]), v["ldy"], v["kind"], p(v["status"]), None)


@pytest.mark.parametrize("over", [
    dict(X=None), dict(A=None), dict(B=None), dict(ids=None), dict(Y=None), dict(status=None), dict(set=False), dict(M=0), dict(K=0), dict(N=0), dict(M=-3), dict(slots=0),
    dict(R=0), dict(ldx=56), dict(lda=56), dict(ldb=8), dict(ldy=120), dict(ldbase=120), dict(kind=2), dict(kind=-1), dict(sa=1016), dict(sb=2040),
    dict(Y=0x100000), dict(Y=0x200000), dict(Y=0x300000 + 3 * 4096 - 16), dict(Y=0x500010), dict(Y=0x500000, ldy=136), dict(Y=0x440000 - 1040, ids=0x440000 - 32),
    dict(Y=0x410000), dict(Y=0x420000),
])
def test_invalid_arguments_are_refused(mx, over):
    assert _call(mx, **over) == mx.MUXQ_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [
    dict(K=60), dict(N=124), dict(R=12, ldb=16), dict(R=136, ldb=136, sa=136 * 64, sb=136 * 128), dict(ldx=68), dict(lda=68, sa=2048), dict(ldb=20, sb=4096), dict(ldy=132),
    dict(ldbase=132), dict(kind=1, ldy=130), dict(sa=1028), dict(sb=2052), dict(X=0x100008), dict(A=0x200008), dict(B=0x300008), dict(Y=0x600008), dict(base=0x500008),
])
def test_unsupported_shapes_are_refused(mx, over):
    assert _call(mx, **over) == mx.MUXQ_ERR_UNSUPPORTED


@pytest.mark.parametrize("at", [0x600000, 0x600000 + 3 * 256 + 252, 0x600000 + 128])
def test_a_status_word_inside_the_result_is_refused(mx, at):
    assert _call(mx, status=at) == mx.MUXQ_ERR_INVALID_ARG


class FakeTensor:
    def __init__(self, shape, stride=None, dtype=F16, device=0):
        self.shape, self.dtype, self._device = shape, dtype, device
        self._stride = stride or tuple(int(torch.tensor(shape[i + 1:]).prod()) if i + 1 < len(shape) else 1 for i in range(len(shape)))

    def get_device(self):
        return self._device

    def stride(self):
        return self._stride

    def data_ptr(self):
        return 0x10000


_FN = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(_CSet), ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                       ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p)


@pytest.fixture
def calls(mx):
    from paper_2604_04701_b200 import binding
    seen = []

    @_FN
    def entry(X, M, K, ldx, s, ids, N, base, ldbase, Y, ldy, kind, status, stream):
        s = s.contents
        seen.append((M, K, ldx, s.lda, s.ldb, s.sa, s.sb, bool(s.scale), bool(s.rank), s.slots, s.max_rank, N, bool(base), ldbase, ldy, kind))
        return 0

    at = ctypes.cast(entry, ctypes.c_void_p).value
    binding._calls.bind(at, at, at, lambda: 0, lambda d: 0, F16, F32, at, at, torch.int32)
    yield binding._calls.adapters, seen
    binding._lib = binding._calls = None
    mx.lib()


def _fake(**over):
    F = FakeTensor
    v = dict(X=F((5, 64)), A=F((3, 16, 64)), B=F((3, 128, 16)), ids=F((5,), dtype=torch.int32), scale=F((3,), dtype=F32), rank=F((3,), dtype=torch.int32), base=F((5, 128)),
             Y=F((5, 128)), status=F((1,), dtype=torch.int32))
    v.update(over)
    return [v[k] for k in ("X", "A", "B", "ids", "scale", "rank", "base", "Y", "status")]


def test_the_binding_passes_shapes_pitches_and_strides(calls):
    f, seen = calls
    F = FakeTensor
    assert f(*_fake()) == 0
    assert f(*_fake(X=F((5, 64), (72, 1)), A=F((3, 16, 64), (5000, 80, 1)), B=F((3, 128, 16), (9000, 32, 1)), Y=F((5, 128), (136, 1), F32),
                    base=None, scale=None, rank=None)) == 0
    big = 1 << 40
    assert f(*_fake(A=F((3, 16, 64), (big, 64, 1)), base=F((5, 128), (256, 1)))) == 0
    assert seen == [(5, 64, 64, 64, 16, 1024, 2048, True, True, 3, 16, 128, True, 128, 128, 0), (5, 64, 72, 80, 32, 5000, 9000, False, False, 3, 16, 128, False, 0, 136, 1),
                    (5, 64, 64, 64, 16, big, 2048, True, True, 3, 16, 128, True, 256, 128, 0)]


@pytest.mark.parametrize("over", [
    dict(X=FakeTensor((5, 64), dtype=F32)), dict(X=FakeTensor((5, 72))), dict(X=FakeTensor((5, 64), (1, 5))), dict(X=FakeTensor((5, 64), device=-1)),
    dict(X=FakeTensor((5, 64), device=1)), dict(A=FakeTensor((3, 16, 64), dtype=F32)), dict(A=FakeTensor((16, 64))), dict(A=FakeTensor((3, 16, 64), device=1)),
    dict(A=FakeTensor((3, 16, 64), (1024, 1, 16))), dict(B=FakeTensor((2, 128, 16))), dict(B=FakeTensor((3, 128, 8))), dict(B=FakeTensor((3, 16, 128), (2048, 1, 16))),
    dict(ids=FakeTensor((4,), dtype=torch.int32)), dict(ids=FakeTensor((5,), dtype=torch.int64)), dict(ids=FakeTensor((5,), (2,), dtype=torch.int32)),
    dict(ids=FakeTensor((5, 1), dtype=torch.int32)), dict(scale=FakeTensor((3,))), dict(scale=FakeTensor((2,), dtype=F32)), dict(rank=FakeTensor((3,), dtype=torch.int64)),
    dict(rank=FakeTensor((4,), dtype=torch.int32)), dict(base=FakeTensor((5, 128), dtype=F32)), dict(base=FakeTensor((4, 128))), dict(Y=FakeTensor((5, 120))),
    dict(Y=FakeTensor((6, 128))), dict(Y=FakeTensor((5, 128), dtype=torch.int32)), dict(status=FakeTensor((1,), dtype=F32)), dict(status=FakeTensor((1,), dtype=torch.int32, device=1)),
])
def test_the_binding_refuses_what_does_not_fit(calls, over):
    f, seen = calls
    with pytest.raises(ValueError):
        f(*_fake(**over))
    assert not seen


# ------------------------------------------------------------------------------------------------ on the GPU
def _inputs(M, K, N, slots, R, ranks, out, seed=0, extra=0, base=True, order="mixed", none=0.2, big=True):
    gen = torch.Generator().manual_seed(1000 * seed + 31 * M + K + N + R)
    X = torch.randn(M, K + extra, generator=gen)
    if big:
        X[:, torch.randperm(K, generator=gen)[:3]] *= 50.0
    A = torch.randn(slots, R, K + extra, generator=gen) / K ** 0.5
    B = torch.randn(slots, N, R + extra, generator=gen) * 0.2
    ids = torch.randint(0, slots, (M,), generator=gen)
    ids[torch.rand(M, generator=gen) < none] = -1
    if order == "runs":
        ids = ids.sort().values
    rank = None if ranks is None else torch.tensor([ranks[i % len(ranks)] for i in range(slots)], dtype=torch.int32)
    A, B = A.half(), B.half()
    if rank is not None:  # what lies beyond a slot's rank is not looked at
        for i in range(slots):
            A[i, int(rank[i]):] = float("nan")
            B[i, :, int(rank[i]):] = float("inf")
    scale = 0.5 + torch.rand(slots, generator=gen)
    b = torch.randn(M, N + extra, generator=gen).to(out) if base else None
    whole = torch.randn(M + 1, N + extra, generator=gen).to(out).cuda()
    dev = lambda t: None if t is None else t.cuda()
    return dict(X=dev(X.half())[:, :K], A=dev(A)[:, :, :K], B=dev(B)[:, :, :R], ids=dev(ids.int()), scale=dev(scale), rank=dev(rank), base=None if b is None else dev(b)[:, :N]), whole


def _run(mx, v, whole):
    M, N = v["X"].shape[0], v["B"].shape[1]
    before, status = whole.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], v["rank"], v["base"], out=whole[:M, :N])
    torch.cuda.synchronize()
    assert int(status) == 0
    assert torch.equal(whole[M:], before[M:]) and torch.equal(whole[:, N:], before[:, N:])  # rows behind the last one, columns behind N
    check(Y, *reference(v["X"], v["A"], v["B"], v["ids"], v["scale"], v["rank"], v["base"]))
    return Y


@pytest.mark.gpu
@pytest.mark.parametrize("out", [F16, F32])
@pytest.mark.parametrize("R,ranks", [(8, None), (8, (1, 3, 8)), (16, (16, 5)), (24, None), (32, (32, 17)), (64, (4, 8, 13, 33, 64)), (72, (65, 72, 2)), (128, None), (128, (127, 100, 1))])
@pytest.mark.parametrize("M", [1, 6, 61, 700])
def test_ranks_and_types(gpu, M, R, ranks, out):
    _run(gpu, *_inputs(M, 264, 200, 5, R, ranks, out, extra=8))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 3, 15, 16, 17, 18, 19, 31, 37, 38, 63, 64, 65, 74, 75, 148, 149, 295, 297, 593, 1003, 1185, 2369, 4800, 9473])
@pytest.mark.parametrize("order,slots", [("mixed", 3), ("runs", 7), ("mixed", 300)])
def test_numbers_of_rows(gpu, M, order, slots):
    """Every size of the windows and of their clusters, with few adapters in a window and with one for every row."""
    _run(gpu, *_inputs(M, 200, 264, slots, 16, (16, 7), F16 if M % 2 else F32, order=order))


@pytest.mark.gpu
@pytest.mark.parametrize("K", [8, 16, 24, 40, 256, 776, 1280, 5120])
@pytest.mark.parametrize("N", [8, 24, 32, 40, 776, 3848])
@pytest.mark.parametrize("M", [1, 20, 130])
def test_channels(gpu, M, K, N):
    _run(gpu, *_inputs(M, K, N, 3, 32, (32, 9, 24), F32))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 33, 650])
def test_without_base_and_without_options(gpu, M):
    mx = gpu
    v, whole = _inputs(M, 264, 136, 4, 16, None, F32, base=False)
    v["scale"] = None
    _run(mx, v, whole)
    v["ids"].fill_(-1)
    assert not _run(mx, v, whole).any()
    v["ids"].fill_(2)
    _run(mx, v, whole)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status).dtype == F16
    assert mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, out_kind=mx.MUXQ_OUT_F32).dtype == F32
    with pytest.raises(mx.MuxqError):
        mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, out_kind=mx.MUXQ_OUT_ACC_I32)


@pytest.mark.gpu
@pytest.mark.parametrize("out", [F16, F32])
@pytest.mark.parametrize("M", [1, 9, 70, 1100])
def test_in_place_and_again(gpu, M, out):
    """base is Y; the same call gives the same bits."""
    mx = gpu
    v, whole = _inputs(M, 520, 392, 6, 24, (24, 11), out, extra=8)
    want = _run(mx, v, whole).clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(3):
        Y = v["base"].clone()
        mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], v["rank"], base=Y, out=Y)
        assert torch.equal(Y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [5, 300])
def test_slots_and_ranks_out_of_range(gpu, M):
    """Reported in the status word; the rows concerned keep base, the others their results."""
    mx = gpu
    v, whole = _inputs(M, 264, 136, 4, 16, (16, 9, 0, 12), F32, none=0.0)
    good = _run(mx, v, whole).clone()  # (rank 0: a slot without an adapter)
    for bad_id, bad_rank in [(4, None), (-2, None), (2 ** 31 - 1, None), (-2 ** 31, None), (None, 17), (None, -1), (None, 2 ** 31 - 1)]:
        ids, rank, status = v["ids"].clone(), v["rank"].clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        if bad_id is not None:
            ids[M // 2] = bad_id
            changed = torch.arange(M, device="cuda") == M // 2
        else:
            ids[M // 2] = 1
            rank[1] = bad_rank
            changed = ids == 1
        Y = mx.muxq_adapters(v["X"], v["A"], v["B"], ids, status, v["scale"], rank, v["base"])
        assert mx.lib().muxq_read_status(ctypes.c_void_p(status.data_ptr()), None) == mx.MUXQ_ERR_INVALID_ARG
        assert torch.equal(Y[changed], v["base"][changed])
        check(Y, *reference(v["X"], v["A"], v["B"], ids, v["scale"], rank, v["base"]))
    assert good.shape == Y.shape
    rank = v["rank"].clone()
    rank[3] = 99  # a slot that no row uses may hold anything
    ids = v["ids"].clone()
    ids[ids == 3] = 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mx.muxq_adapters(v["X"], v["A"], v["B"], ids, status, v["scale"], rank, v["base"])
    assert int(status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("size", [1e-7, 1e-3, 1.0, 6e4])
def test_magnitudes(gpu, size, M):
    """Rows of X whose products leave the range of fp16 in either direction."""
    mx = gpu
    v, whole = _inputs(M, 264, 136, 3, 16, None, F32, big=False)
    v["X"] = (v["X"].float().clamp(-1, 1) * size).half()
    v["X"][0] = 0.0
    v["base"] = None
    _run(mx, v, whole)
    v["A"] = v["A"] * 16 if size > 1 else v["A"]
    _run(mx, v, whole)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [6, 90, 1300])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_request_that_is_not_finite_stays_alone(gpu, value, M):
    """A row of X, and an adapter, that hold no numbers: every other row keeps its bits."""
    mx = gpu
    v, whole = _inputs(M, 264, 136, 4, 16, None, F32, none=0.1)
    good = _run(mx, v, whole).clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    row = int((v["ids"] >= 0).nonzero()[0])
    X = v["X"].clone()
    X[row, 77] = value
    Y = mx.muxq_adapters(X, v["A"], v["B"], v["ids"], status, v["scale"], None, v["base"])
    keep = torch.arange(M, device="cuda") != row
    assert torch.equal(Y[keep], good[keep])
    for which in ("A", "B"):
        w = {k: v[k].clone() for k in ("A", "B")}
        w[which][2, 5, 7] = value
        Y = mx.muxq_adapters(v["X"], w["A"], w["B"], v["ids"], status, v["scale"], None, v["base"])
        assert torch.equal(Y[v["ids"] != 2], good[v["ids"] != 2])
    assert int(status) == 0


def _runs(gen, M, slots, lengths):
    """Slots of M rows in runs of the given lengths, -1 among them."""
    ids, i = torch.empty(M, dtype=torch.int64), 0
    at = 0
    while at < M:
        n = lengths[i % len(lengths)]
        ids[at:at + n] = int(torch.randint(-1, slots, (1,), generator=gen)) if i % 5 else i % slots
        at, i = at + n, i + 1
    return ids.int().cuda()


# windows of 128 rows with one adapter, with two to four, with more than any window may have, and all of these in one batch
LENGTHS = {"long": (1000, 333), "short": (70, 61, 90, 20), "few": (33, 32, 40), "mixed": (5, 600, 40, 129, 1, 31, 32, 300)}


@pytest.mark.gpu
@pytest.mark.parametrize("out", [F16, F32])
@pytest.mark.parametrize("R,ranks", [(8, None), (16, (16, 0)), (16, (16, 7, 16)), (24, (24, 16)), (32, (32, 16)), (64, (64, 16, 48)), (72, (72, 64)), (128, None), (128, (128, 100, 16, 96))])
@pytest.mark.parametrize("lengths", sorted(LENGTHS))
def test_long_inputs(gpu, lengths, R, ranks, out):
    v, whole = _inputs(1500, 264, 200, 5, R, ranks, out, extra=8)
    v["ids"] = _runs(torch.Generator().manual_seed(R), 1500, 5, LENGTHS[lengths])
    _run(gpu, v, whole)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1023, 1024, 1025, 2047, 4097])
@pytest.mark.parametrize("K,N", [(8, 8), (24, 72), (200, 64), (1288, 136), (64, 1992), (776, 520)])
def test_long_inputs_of_all_sizes(gpu, M, K, N):
    """Rows that end inside a window, K and N inside a step; base is Y."""
    mx = gpu
    v, whole = _inputs(M, K, N, 3, 16, (16, 16, 9), F32)
    v["ids"] = _runs(torch.Generator().manual_seed(N), M, 3, (400, 90, 129))
    want = _run(mx, v, whole).clone()
    Y, status = v["base"].clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(2):
        Y.copy_(v["base"])
        mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], v["rank"], base=Y, out=Y)
        assert torch.equal(Y, want)
    v["base"] = None
    _run(mx, v, whole)


@pytest.mark.gpu
def test_long_inputs_slots_and_ranks_out_of_range(gpu):
    mx = gpu
    v, whole = _inputs(2000, 264, 136, 4, 16, (16, 16, 0, 16), F32)
    v["ids"] = _runs(torch.Generator().manual_seed(3), 2000, 4, (500, 90, 300))
    _run(mx, v, whole)
    for bad_id, bad_rank in [(4, None), (-2, None), (2 ** 31 - 1, None), (-2 ** 31, None), (None, 17), (None, -1)]:
        ids, rank, status = v["ids"].clone(), v["rank"].clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        if bad_id is not None:
            ids[700] = bad_id
        else:
            ids[700] = 1
            rank[1] = bad_rank
        Y = mx.muxq_adapters(v["X"], v["A"], v["B"], ids, status, v["scale"], rank, v["base"])
        assert int(status) == mx.MUXQ_ERR_INVALID_ARG
        changed = torch.arange(2000, device="cuda") == 700 if bad_id is not None else ids == 1
        assert torch.equal(Y[changed], v["base"][changed])
        check(Y, *reference(v["X"], v["A"], v["B"], ids, v["scale"], rank, v["base"]))


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_long_inputs_that_are_not_finite_stay_alone(gpu, value):
    """Adapters of one window do not reach each other's rows, whatever they hold."""
    mx = gpu
    v, whole = _inputs(1300, 264, 136, 4, 16, None, F32)
    v["ids"] = _runs(torch.Generator().manual_seed(5), 1300, 4, (50, 70, 128, 30))
    good, status = _run(mx, v, whole).clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    row = int((v["ids"] >= 0).nonzero()[0])
    X = v["X"].clone()
    X[row, 77] = value
    Y = mx.muxq_adapters(X, v["A"], v["B"], v["ids"], status, v["scale"], None, v["base"])
    keep = torch.arange(1300, device="cuda") != row
    assert torch.equal(Y[keep], good[keep])
    for which in ("A", "B"):
        w = {k: v[k].clone() for k in ("A", "B")}
        w[which][2, 5, 7] = value
        Y = mx.muxq_adapters(v["X"], w["A"], w["B"], v["ids"], status, v["scale"], None, v["base"])
        assert torch.equal(Y[v["ids"] != 2], good[v["ids"] != 2])
    base = v["base"].clone()
    base[::7, 3] = value
    Y = mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], None, base)
    keep = torch.ones(1300, 136, dtype=torch.bool, device="cuda")
    keep[::7, 3] = False
    assert torch.equal(Y[keep], good[keep]) and not torch.isfinite(Y[~keep]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("M,names", [(1, ["k_adapters"]), (1023, ["k_adapters"]), (1024, ["k_adapter_tiles", "k_adapters"])])
def test_which_kernels_run(gpu, M, names):
    from conftest import kernels_launched
    v, whole = _inputs(M, 264, 200, 5, 16, (16, 7), F16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    call = lambda: gpu.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], v["rank"], v["base"], out=whole[:M, :200])
    call()
    torch.cuda.synchronize()
    ran = [name for name, _ in kernels_launched(call)]
    assert len(ran) == len(names) and all(n in r for n, r in zip(names, ran)), ran


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 200, 1500])
def test_two_calls_at_once(gpu, M):
    """No workspace: calls on two streams do not disturb each other."""
    mx = gpu
    u, whole = _inputs(M, 776, 392, 6, 24, (24, 11, 16), F32)
    v, _ = _inputs(M, 776, 392, 6, 24, (24, 11, 16), F32, seed=3)
    u["ids"] = v["ids"] = _runs(torch.Generator().manual_seed(1), M, 6, (300, 200, 70))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = lambda w: (w["X"], w["A"], w["B"], w["ids"], status, w["scale"], w["rank"], w["base"])
    want = [mx.muxq_adapters(*args(w)).clone() for w in (u, v)]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(want[0]) for _ in range(2)]
    for _ in range(20):
        for k, w in enumerate((u, v)):
            with torch.cuda.stream(side[k]):
                mx.muxq_adapters(*args(w), out=outs[k])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]) and int(status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("R,ranks", [(64, (5, 33, 64, 17)), (40, (37,)), (128, (100, 65))])
@pytest.mark.parametrize("lengths", ["long", "short"])
def test_long_inputs_whose_ranks_end_inside_a_step(gpu, lengths, R, ranks):
    """What stands beyond such a rank is no number (see _inputs), in one window beside adapters of other ranks."""
    for N in (72, 520, 1992):
        v, whole = _inputs(1400, 200, N, 4, R, ranks, F32)
        v["ids"] = _runs(torch.Generator().manual_seed(N), 1400, 4, LENGTHS[lengths])
        _run(gpu, v, whole)


@pytest.mark.gpu
def test_long_inputs_time_out(gpu):
    """A wait that runs out (the loads of a part of K are left out by a test hook) ends the kernel with a status; the next call is right."""
    mx = gpu
    v, whole = _inputs(1500, 776, 200, 2, 32, None, F16)
    v["ids"].fill_(1)
    want = _run(mx, v, whole).clone()
    before = whole.clone()
    for chunk in (1, 5, 12):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        mx.muxq_test_hooks(spin_limit=20000, gemm_skip_k_block=chunk)
        try:
            mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], None, v["base"], out=whole[:1500, :200])
            torch.cuda.synchronize()
        finally:
            mx.muxq_test_hooks()
        assert int(status) == mx.MUXQ_ERR_TIMEOUT
        assert torch.equal(whole[1500:], before[1500:])
        assert torch.equal(_run(mx, v, whole), want)


@pytest.mark.gpu
def test_an_adapter_loaded_ahead_of_the_call(gpu):
    """Slots are rewritten and rows reassigned between the replays of one graph, and by work directly ahead on the stream."""
    mx = gpu
    v, whole = _inputs(24, 264, 136, 4, 16, None, F16)
    w, _ = _inputs(24, 264, 136, 4, 16, None, F16, seed=5)
    status, side, Y = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cuda.Stream(), torch.empty_like(v["base"])
    side.wait_stream(torch.cuda.current_stream())
    args = lambda u: (u["X"], u["A"], u["B"], u["ids"], status, u["scale"], None, u["base"])
    with torch.cuda.stream(side):
        want_v, want_w = mx.muxq_adapters(*args(v)).clone(), mx.muxq_adapters(*args(w)).clone()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            mx.muxq_adapters(*args(v), out=Y)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, want_v)
    for k in ("X", "A", "B", "ids", "scale", "base"):
        v[k].copy_(w[k])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, want_w)


@pytest.mark.gpu
def test_offsets_beyond_32_bits(gpu):
    """Slots a gigabyte of elements apart."""
    mx = gpu
    v, whole = _inputs(9, 64, 136, 3, 16, None, F32)
    far = torch.empty((2 << 30) + 16 * 64, dtype=F16, device="cuda").as_strided((3, 16, 64), (1 << 30, 64, 1))
    far.copy_(v["A"])
    v["A"] = far
    _run(mx, v, whole)
    rows = torch.empty((2 << 30) + 136, dtype=F16, device="cuda").as_strided((3, 136), (1 << 30, 1))
    v, _ = _inputs(3, 64, 136, 3, 16, None, F16, none=0.0)
    rows.copy_(v["base"])
    v["base"] = rows
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], None, v["base"])
    check(Y, *reference(v["X"], v["A"], v["B"], v["ids"], v["scale"], None, v["base"]))


# ------------------------------------------------------------------------------------------------ beside muxq_linear
class _Operand(FakeTensor):
    is_cuda = True

    def __init__(self, *a, at=0x100000, **k):
        super().__init__(*a, **k)
        self.at = at

    def data_ptr(self):
        return self.at

    def numel(self):
        return int(torch.tensor(self.shape).prod())

    def is_contiguous(self):
        return True


_LINEAR_FN = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p)


@pytest.fixture
def layer(mx):
    """(muxq_linear with adapters on stand-ins for tensors, what was launched); the entry points are stand-ins too, but for the check"""
    from paper_2604_04701_b200 import binding
    launched = []

    @_LINEAR_FN
    def linear(*a):
        launched.append("linear")
        return 0

    @_FN
    def adapters(*a):
        launched.append("adapters")
        return 0

    L = mx.lib()
    at = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    binding._calls.bind(at(linear), at(linear), at(linear), lambda: 0, lambda d: 0, F16, F32, at(adapters), at(adapters), torch.int32, at(L.muxq_adapters_check))
    O = _Operand
    i32 = torch.int32

    def call(out_kind=None, **over):
        v = dict(X=O((5, 64), at=0x100000), out=O((5, 128), at=0x600000), A=O((3, 16, 64), at=0x200000), B=O((3, 128, 16), at=0x300000), row_slot=O((5,), dtype=i32, at=0x400000),
                 scale=O((3,), dtype=F32, at=0x410000), rank=O((3,), dtype=i32, at=0x420000))
        v.update(over)
        ws = type("Ws", (), dict(buf=O((4096,), dtype=torch.uint8), status=O((1,), dtype=i32, at=0x440000)))
        return mx.muxq_linear(v["X"], O((128, 64), dtype=torch.int8), O((1,), dtype=F32), mx.MuxqParams(), ws, mx.MUXQ_OUT_F16 if out_kind is None else out_kind, out=v["out"],
                              adapters=mx.Adapters(v["A"], v["B"], v["row_slot"], v["scale"], v["rank"]))

    yield call, launched
    binding._lib = binding._calls = None
    mx.lib()


def test_the_layer_runs_with_its_adapters_behind_it(layer):
    call, launched = layer
    call()
    assert launched == ["linear", "adapters"]


@pytest.mark.parametrize("over", [
    dict(A=_Operand((3, 16, 72))), dict(B=_Operand((3, 120, 16))), dict(B=_Operand((2, 128, 16))), dict(A=_Operand((3, 16, 64), dtype=F32)), dict(A=_Operand((16, 64))),
    dict(A=_Operand((3, 16, 64), device=1)), dict(row_slot=_Operand((4,), dtype=torch.int32)), dict(row_slot=_Operand((5,), dtype=torch.int64)), dict(scale=_Operand((2,), dtype=F32)),
    dict(rank=_Operand((3,), dtype=torch.int64)), dict(out=_Operand((6, 128))),
    dict(out=_Operand((5, 128), dtype=F32)), dict(out_kind=1),  # out is not of out_kind
])
def test_adapters_that_do_not_fit_are_refused_before_the_layer_runs(layer, over):
    call, launched = layer
    with pytest.raises(ValueError):
        call(**over)
    assert not launched


@pytest.mark.parametrize("over,code", [
    (dict(out=_Operand((5, 128), at=0x100000)), 1),  # over X
    (dict(A=_Operand((3, 16, 64), (512, 64, 1), at=0x200000)), 1), (dict(A=_Operand((3, 16, 64), at=0x200008)), 2), (dict(out=_Operand((5, 128), (132, 1), at=0x600000)), 2),
    (dict(A=_Operand((3, 12, 64), at=0x200000), B=_Operand((3, 128, 12), (2048, 16, 1), at=0x300000)), 2), (dict(out_kind=2), 1),
])
def test_adapters_that_the_library_refuses_are_refused_before_the_layer_runs(mx, layer, over, code):
    call, launched = layer
    with pytest.raises(mx.MuxqError) as e:
        call(**over)
    assert e.value.status == code and not launched


def test_the_check_says_what_the_call_would(mx):
    """muxq_adapters_check launches nothing: a call that would be taken can be asked about without a device."""
    p = ctypes.c_void_p

    def check(**over):
        v = dict(Y=0x600000, ldy=128, K=64, ldbase=128)
        v.update(over)
        s = _CSet(0x200000, 0x300000, 64, 16, 1024, 2048, 0x410000, 0x420000, 3, 16)
        return mx.lib().muxq_adapters_check(p(0x100000), 4, v["K"], 64, ctypes.byref(s), p(0x430000), 128, p(0x500000), v["ldbase"], p(v["Y"]), v["ldy"], 0, p(0x440000))

    assert check() == mx.MUXQ_OK and check(Y=0x500000) == mx.MUXQ_OK
    assert check(Y=0x500010) == check(ldbase=120) == check(Y=0x100000) == mx.MUXQ_ERR_INVALID_ARG
    assert check(K=60) == check(ldy=132) == mx.MUXQ_ERR_UNSUPPORTED


@pytest.mark.gpu
def test_a_refused_layer_leaves_its_result_alone(gpu):
    mx = gpu
    gen = torch.Generator().manual_seed(1)
    K, N, M = 256, 640, 16
    p = mx.MuxqParams()
    w_q, s_w = mx.muxq_quantize((torch.randn(K, N, generator=gen) * 0.03).half().cuda(), p, True, mx.Workspace(mx.muxq_small_workspace_bytes(N)))
    ws = mx.Workspace(mx.muxq_workspace_bytes(M, K, N, p))
    v, whole = _inputs(M, K, N, 3, 16, None, F16)
    out = whole[:M]
    before = out.clone()
    good = mx.Adapters(v["A"], v["B"], v["ids"], v["scale"])
    for bad, error in ((good._replace(A=v["A"][:, :8]), ValueError), (good._replace(row_slot=v["ids"][:5]), ValueError), (good._replace(B=v["B"][:, :128]), ValueError)):
        with pytest.raises(error):
            mx.muxq_linear(v["X"], w_q, s_w, p, ws, mx.MUXQ_OUT_F16, out=out, adapters=bad)
        torch.cuda.synchronize()
        assert torch.equal(out, before)
    alone = mx.muxq_linear(v["X"], w_q, s_w, p, ws, mx.MUXQ_OUT_F16)
    mx.muxq_linear(v["X"], w_q, s_w, p, ws, mx.MUXQ_OUT_F16, out=out, adapters=good)
    assert mx.muxq_read_status(ws) == mx.MUXQ_OK
    check(out, *reference(v["X"], v["A"], v["B"], v["ids"], v["scale"], None, alone))


def test_operands_beside_the_result_in_one_wider_matrix(mx):
    """Columns that lie side by side do not overlap, be it those of every row, of every second one or of one."""
    p = ctypes.c_void_p

    def check(ldy=256, **over):  # Y: four rows of 256 bytes, 512 apart
        v = dict(scale=0x410000, rank=0x420000, base=0x500000, ldbase=128, status=0x440000, X=0x100000, ldx=64)
        v.update(over)
        s = _CSet(0x200000, 0x300000, 64, 16, 1024, 2048, v["scale"], v["rank"], 3, 16)
        return mx.lib().muxq_adapters_check(p(v["X"]), 4, 64, v["ldx"], ctypes.byref(s), p(0x430000), 128, p(v["base"]), v["ldbase"], p(0x600000), ldy, 0, p(v["status"]))

    Y = 0x600000
    for free in (dict(scale=Y + 256), dict(rank=Y + 500), dict(status=Y + 2 * 512 + 400), dict(base=Y + 256, ldbase=256), dict(base=Y + 256, ldbase=512), dict(base=Y + 512 + 256, ldbase=768),
                 dict(X=Y + 256, ldx=1024), dict(X=Y - 128, ldx=256), dict(scale=Y + 3 * 512 + 256)):
        assert check(**free) == mx.MUXQ_OK, free
    for over in (dict(scale=Y + 248), dict(scale=Y + 504), dict(rank=Y + 512), dict(status=Y + 2 * 512 + 252), dict(base=Y + 240, ldbase=512), dict(base=Y + 272, ldbase=512),
                 dict(base=Y + 256, ldbase=384), dict(X=Y + 240, ldx=1024), dict(X=Y - 112, ldx=256), dict(X=Y + 512 - 16, ldx=512)):
        assert check(**over) == mx.MUXQ_ERR_INVALID_ARG, over


@pytest.mark.parametrize("dtype,out_kind", [(F32, 0), (F16, 1), (F16, 2), (torch.int32, 2)])
def test_a_result_of_another_type_than_out_kind_is_refused(mx, dtype, out_kind):
    t = lambda *s: torch.zeros(*s, dtype=F16)
    with pytest.raises((ValueError, mx.MuxqError), match="out_kind|invalid"):
        mx.muxq_adapters(t(5, 64), t(3, 16, 64), t(3, 128, 16), torch.zeros(5, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), out_kind=out_kind,
                         out=torch.zeros(5, 128, dtype=dtype))
