"""muxq_residual_norm: h = R + alpha * gate * post(Y), x = pre(h), against the formulas in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32 relative to the value.  A sum over a row is a tree of at most 12 additions in a thread, 5 in a
warp and 16 over the warps, so its relative error is at most 33 u of the sum of magnitudes; with the division by D the mean is off by at
most 36 u mean|v|.  The mean square has two roundings more per term, and the root halves its relative error: 1 / sqrt is off by at most 22 u
relatively (the error of the mean enters the squares in second order).  Weight, bias, gate, alpha and the sum with R are at most 6 roundings.  Together: 64 u times
the magnitudes that each of them multiplies.  What x inherits from the error of h follows from the derivative of the norm:
r |w| (e + mean e + |h - mu| r rms(e)).  A result in fp16 is off by half a step more, 2^-11 of the value, or 2^-25 where it is subnormal."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

U = 2.0 ** -24
NONE, RMS, LAYER = 0, 1, 2


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


# ------------------------------------------------------------------------------------------------ the formulas in 64 bits
def _norm64(v, e, kind, weight, bias, eps):
    """(norm of v, bound of its error when v is off by at most e)"""
    if kind == NONE:
        return v, e
    w = torch.ones(v.shape[1], dtype=torch.float64) if weight is None else weight.double().cpu()
    b = torch.zeros(v.shape[1], dtype=torch.float64) if bias is None else bias.double().cpu()
    mu = v.mean(1, keepdim=True) if kind == LAYER else torch.zeros(v.shape[0], 1, dtype=torch.float64)
    d = v - mu
    r = ((d * d).mean(1, keepdim=True) + eps) ** -0.5
    out = d * r * w + b
    own = 64 * U * (w.abs() * r * (v.abs() + v.abs().mean(1, keepdim=True)) + b.abs())
    inherited = w.abs() * r * (e + e.mean(1, keepdim=True) + d.abs() * r * (e * e).mean(1, keepdim=True).sqrt())
    return out, own + inherited


def _half_step(v, dtype):
    return v.abs() * 2.0 ** -11 + 2.0 ** -25 if dtype == torch.float16 else v.abs() * U


def reference(R, Y, pre, post, gate, group, alpha):
    """(h, error of h before it is rounded, x, error of x before it is rounded)"""
    alpha = float(torch.tensor(alpha, dtype=torch.float32))
    some = Y if R is None else R
    h = torch.zeros(some.shape, dtype=torch.float64) if R is None else R.double().cpu()
    e = torch.zeros_like(h)
    if Y is not None:
        y = Y.double().cpu()
        v, ev = _norm64(y, torch.zeros_like(y), *(post[0], post[1], post[2], float(torch.tensor(post[3], dtype=torch.float32))) if post else (NONE, None, None, 0))
        g = torch.ones_like(v)
        if gate is not None:
            g = gate.double().cpu()
            g = g.expand_as(v) if g.dim() == 1 else g.repeat_interleave(group, 0)[:v.shape[0]]
        e = (alpha * g).abs() * ev + 8 * U * (h.abs() + (alpha * g * v).abs())
        h = h + alpha * g * v
    x, ex = (h, e) if pre is None else _norm64(h, e, pre[0], pre[1], pre[2], float(torch.tensor(pre[3], dtype=torch.float32)))
    return h, e, x, ex


def check(out, dtype, want, err, what):
    off = (out.double().cpu() - want).abs()
    tol = err + _half_step(want.abs() + err, dtype)
    assert torch.isfinite(out).all(), what
    assert (off <= tol).all(), (what, float((off / tol).max()))


# ------------------------------------------------------------------------------------------------ refusals, without a GPU
class _CNorm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


def _call(mx, **over):
    """A call that would be valid but for what `over` says; its pointers are never dereferenced, so everything here has to be refused."""
    v = dict(R=0x100000, ldr=64, rk=1, Y=0x200000, ldy=64, yk=0, post=None, g=None, ldg=0, gk=1, group=0, alpha=1.0, pre=_CNorm(2, 1e-5, 0x300000, 0x301000),
             M=4, D=64, H=0x400000, ldh=64, X=0x500000, ldx=64)
    v.update(over)
    p = lambda a: None if a is None else ctypes.c_void_p(a)
    n = lambda a: None if a is None else ctypes.byref(a)
    return mx.lib().muxq_residual_norm(p(v["R"]), v["ldr"], v["rk"], p(v["Y"]), v["ldy"], v["yk"], n(v["post"]), p(v["g"]), v["ldg"], v["gk"], v["group"],
                                       v["alpha"], n(v["pre"]), v["M"], v["D"], p(v["H"]), v["ldh"], p(v["X"]), v["ldx"], None)


@pytest.mark.parametrize("over", [
    dict(R=None, Y=None), dict(H=None, X=None), dict(M=0), dict(D=0), dict(M=-1), dict(rk=2), dict(yk=2), dict(rk=-1), dict(ldr=56), dict(ldy=56), dict(ldh=56),
    dict(ldx=56), dict(g=0x600000, gk=2), dict(g=0x600000, group=-1), dict(g=0x600000, group=1, ldg=56), dict(alpha=float("nan")), dict(alpha=float("inf")),
    dict(pre=_CNorm(3, 1e-5, None, None)), dict(pre=_CNorm(1, 0.0, None, None)), dict(pre=_CNorm(1, -1.0, None, None)),
    dict(pre=_CNorm(1, float("inf"), None, None)), dict(pre=_CNorm(1, float("nan"), None, None)), dict(post=_CNorm(-1, 1e-5, None, None)),
    dict(pre=_CNorm(0, 1e-5, 0x300000, None)), dict(post=_CNorm(0, 1e-5, None, 0x300000)),
    dict(Y=None, g=0x600000), dict(Y=None, post=_CNorm(1, 1e-5, None, None)),
    # results over what is read, or over each other
    dict(X=0x200000), dict(X=0x100000), dict(X=0x400000), dict(H=0x200000), dict(H=0x100010), dict(H=0x100000, ldh=72), dict(X=0x200000 + 3 * 128),
    dict(H=0x300000), dict(X=0x301000 - 256), dict(g=0x400000), dict(g=0x500080, group=1, ldg=64),
])
def test_invalid_arguments_are_refused(mx, over):
    assert _call(mx, **over) == mx.MUXQ_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [
    dict(D=60, ldr=64), dict(D=16392, ldr=16392, ldy=16392, ldh=16392, ldx=16392, R=0x10000000, Y=0x20000000, H=0x30000000, X=0x40000000), dict(R=0x100008), dict(Y=0x200002),
    dict(H=0x400004), dict(X=0x500008), dict(g=0x600004), dict(pre=_CNorm(1, 1e-5, 0x300004, None)), dict(pre=_CNorm(2, 1e-5, None, 0x300008)),
    dict(ldr=66), dict(ldy=68), dict(ldh=67), dict(ldx=68), dict(g=0x600000, gk=0, group=1, ldg=68),
])
def test_unsupported_shapes_are_refused(mx, over):
    assert _call(mx, **over) == mx.MUXQ_ERR_UNSUPPORTED


class FakeTensor:
    def __init__(self, shape, stride=None, dtype=torch.float16, device=0, at=0x10000):
        self.shape, self.dtype, self._device, self._at = shape, dtype, device, at
        self._stride = stride or tuple(int(torch.tensor(shape[i + 1:]).prod()) if i + 1 < len(shape) else 1 for i in range(len(shape)))

    def get_device(self):
        return self._device

    def stride(self):
        return self._stride

    def data_ptr(self):
        return self._at


_FN = ctypes.CFUNCTYPE(ctypes.c_int, *([ctypes.c_void_p, ctypes.c_int, ctypes.c_int] * 2), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                       ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                       ctypes.c_int, ctypes.c_void_p)


@pytest.fixture
def calls(mx):
    from paper_2604_04701_b200 import binding
    seen = []

    @_FN
    def entry(R, ldr, rk, Y, ldy, yk, post, g, ldg, gk, group, alpha, pre, M, D, H, ldh, X, ldx, s):
        seen.append((bool(R), ldr, rk, bool(Y), ldy, yk, bool(g), ldg, gk, group, alpha, M, D, bool(H), ldh, bool(X), ldx))
        return 0

    at = ctypes.cast(entry, ctypes.c_void_p).value
    binding._calls.bind(at, at, at, lambda: 0, lambda d: 0, torch.float16, torch.float32, at)
    yield binding._calls.residual_norm, seen
    binding._lib = binding._calls = None
    mx.lib()


def test_the_binding_passes_shapes_pitches_and_types(calls, mx):
    f, seen = calls
    F = FakeTensor
    n = mx.Norm(LAYER, F((64,), dtype=torch.float32), None)
    assert f(F((5, 64), (80, 1), torch.float32), F((5, 64), (96, 1)), n, None, F((2, 64), (72, 1)), 3, 0.5, F((5, 64), dtype=torch.float32), F((5, 64))) == 0
    assert f(None, F((1, 64), (7, 1)), None, n, F((64,), dtype=torch.float32), 1, 2.0, F((1, 64)), None) == 0  # the pitch of one row says nothing
    assert f(F((5, 64)), None, n, None, None, 1, 1.0, None, F((5, 64))) == 0
    assert seen == [(True, 80, 1, True, 96, 0, True, 72, 0, 3, 0.5, 5, 64, True, 64, True, 64),
                    (False, 64, 0, True, 64, 0, True, 64, 1, 0, 2.0, 1, 64, True, 64, False, 0),
                    (True, 64, 0, False, 0, 0, False, 0, 0, 1, 1.0, 5, 64, False, 0, True, 64)]


def test_the_binding_refuses_what_does_not_fit(calls, mx):
    f, seen = calls
    F, n = FakeTensor, mx.Norm(RMS)
    R, Y, X = F((5, 64)), F((5, 64)), F((5, 64))
    f32 = torch.float32
    for bad in [(None, None, n, None, None, 1, 1.0, None, X), (F((5, 64), device=-1), Y, n, None, None, 1, 1.0, R, X), (F((5, 64), device=1), Y, n, None, None, 1, 1.0, R, X),
                (R, F((5, 64), device=1), n, None, None, 1, 1.0, R, X), (F((5, 64), dtype=torch.bfloat16), Y, n, None, None, 1, 1.0, R, X),
                (R, F((4, 64)), n, None, None, 1, 1.0, R, X), (R, F((5, 72)), n, None, None, 1, 1.0, R, X), (F((5, 64), (1, 5)), Y, n, None, None, 1, 1.0, R, X),
                (R, Y, n, None, None, 1, 1.0, F((5, 64), dtype=f32), X), (R, Y, n, None, None, 1, 1.0, R, F((5, 64), dtype=f32)), (R, Y, n, None, None, 1, 1.0, R, F((6, 64))),
                (R, Y, mx.Norm(RMS, F((64,))), None, None, 1, 1.0, R, X), (R, Y, mx.Norm(RMS, F((32,), dtype=f32)), None, None, 1, 1.0, R, X),
                (R, Y, mx.Norm(RMS, F((64,), (2,), dtype=f32)), None, None, 1, 1.0, R, X), (R, Y, n, None, F((4, 64)), 1, 1.0, R, X), (R, Y, n, None, F((5, 64)), 2, 1.0, R, X),
                (R, Y, n, None, F((5, 64)), 0, 1.0, R, X), (R, Y, n, None, F((32,)), 1, 1.0, R, X), (R, Y, n, None, F((1, 5, 64)), 1, 1.0, R, X),
                (F((5, 8, 64)), Y, n, None, None, 1, 1.0, R, X), (F((64,)), Y, n, None, None, 1, 1.0, R, X), (R, Y, (1, 2), None, None, 1, 1.0, R, X)]:
        with pytest.raises(ValueError):
            f(*bad)
    with pytest.raises(ValueError):
        f(F(()), Y, n, None, None, 1, 1.0, R, X)
    assert not seen


# ------------------------------------------------------------------------------------------------ on the GPU
def _wide(rows, cols, extra, dtype, gen, scale=1.0, shift=0.0):
    """[rows, cols] as columns of a wider matrix, and that matrix."""
    whole = (torch.randn(rows + 2, cols + extra, generator=gen) * scale + shift).to(dtype).cuda()
    return whole[:rows, :cols], whole


def _vec(gen, D, around=1.0):
    return (around + 0.3 * torch.randn(D, generator=gen)).cuda()


def _run(mx, M, D, res, blk, post, pre, gate, group=1, alpha=0.7, extra=0, seed=0, scale=1.0, shift=0.0, in_place=False):
    gen = torch.Generator().manual_seed(seed + 7 * M + D)
    R = _wide(M, D, extra, res, gen, 3.0 * scale, shift)[0] if res else None
    Y = _wide(M, D, extra, blk, gen, scale, shift)[0] if blk else None
    norms = []
    for kind in (pre, post):
        norms.append(None if kind == NONE else mx.Norm(kind, _vec(gen, D), _vec(gen, D, 0.0) if kind == LAYER else None, 1e-5))
    g = None
    if gate == "channel":
        g = _vec(gen, D, 0.5)
    elif gate:
        g = _wide(-(-M // group), D, extra, torch.float16 if gate == "f16" else torch.float32, gen, 0.5)[0]
    kind = res or torch.float32
    want = reference(R, Y, norms[0], norms[1], g, group, alpha)
    h_out = H_whole = None
    if Y is not None:
        if in_place:
            h_out, H_whole = R, None
        else:
            h_out, H_whole = _wide(M, D, extra, kind, gen)
    x_out, X_whole = _wide(M, D, extra, torch.float16, gen)
    before = [w.clone() for w in (H_whole, X_whole) if w is not None]
    H, X = mx.muxq_residual_norm(R, Y, norms[0], post=norms[1], gate=g, gate_group=group, scale=alpha, H=h_out, X=x_out)
    torch.cuda.synchronize()
    h, e, x, ex = want
    if Y is not None:
        check(H, kind, h, e, "h")
    check(X, torch.float16, x, ex, "x")
    for w, b in zip([w for w in (H_whole, X_whole) if w is not None], before):  # rows behind the last one, columns behind D
        assert torch.equal(w[M:], b[M:]) and torch.equal(w[:, D:], b[:, D:])
    return H, X


F16, F32 = torch.float16, torch.float32


@pytest.mark.gpu
@pytest.mark.parametrize("res", [F16, F32])
@pytest.mark.parametrize("blk", [F16, F32, None])
@pytest.mark.parametrize("post,pre", [(NONE, LAYER), (RMS, RMS), (LAYER, LAYER), (NONE, NONE), (RMS, NONE), (LAYER, RMS)])
@pytest.mark.parametrize("M,D", [(1, 768), (7, 1040), (701, 136)])
def test_types_and_kinds(gpu, M, D, post, pre, blk, res):
    if blk is None and post != NONE:
        post = NONE
    _run(gpu, M, D, res, blk, post, pre, "channel" if blk else None, extra=24)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [8, 16, 24, 120, 128, 136, 256, 384, 392, 640, 768, 1000, 1024, 1280, 1288, 1600, 2048, 2560, 3840, 4096, 5120, 5128, 8192, 12296, 16384])
@pytest.mark.parametrize("M", [1, 2, 593, 1801])
def test_widths(gpu, M, D):
    """Every number of channels a thread and threads a row, for few rows and many."""
    if M * D > 6_000_000:
        M = 6_000_000 // D
    _run(gpu, M, D, F32, F16, RMS, LAYER, None)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["channel", "f16", "f32"])
@pytest.mark.parametrize("M,group", [(1, 1), (6, 1), (6, 3), (7, 3), (5, 9), (900, 1), (901, 128)])
def test_gates(gpu, M, group, gate):
    _run(gpu, M, 776, F16, F32, RMS, RMS, gate, group=group, extra=8)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 1200])
@pytest.mark.parametrize("res", [F16, F32])
def test_the_stream_in_place(gpu, res, M):
    _run(gpu, M, 1280, res, F16, LAYER, LAYER, "f16", in_place=True, extra=16)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [4, 800])
def test_no_stream(gpu, M):
    """R absent: the second term alone."""
    _run(gpu, M, 776, None, F16, RMS, LAYER, "channel")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("scale,shift", [(1.0, 1000.0), (1e-4, 0.0), (1e-4, 1.0), (1e6, 0.0), (1e-12, 0.0), (1e12, 0.0)])
def test_magnitudes(gpu, scale, shift, kind):
    """A mean far from zero, values whose squares are small beside eps or are lost, and large ones."""
    for M in (5, 700):
        _run(gpu, M, 1280, F32, F32, kind, kind, None, scale=scale, shift=shift)


@pytest.mark.gpu
def test_rows_of_zeros_and_of_one_value(gpu):
    mx = gpu
    R = torch.zeros(4, 256, device="cuda")
    R[1] = 5.0
    R[2, 17] = 2.0
    w, b = torch.full((256,), 2.0, device="cuda"), torch.full((256,), 0.5, device="cuda")
    _, x = mx.muxq_residual_norm(R, None, mx.Norm(LAYER, w, b))
    assert torch.equal(x[0], torch.full_like(x[0], 0.5)) and torch.equal(x[1], torch.full_like(x[1], 0.5)) and torch.equal(x[3], x[0])
    _, x = mx.muxq_residual_norm(R, None, mx.Norm(RMS, w))
    assert torch.equal(x[0], torch.zeros_like(x[0])) and float(x[2, 17]) == pytest.approx(2 * 2 / (4 / 256 + 1e-5) ** 0.5, rel=2 ** -11)
    _, x = mx.muxq_residual_norm(R, None, None)
    assert torch.equal(x, R.half())


@pytest.mark.gpu
@pytest.mark.parametrize("M", [9, 900])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 3e38])
def test_a_row_that_is_not_finite_stays_alone(gpu, value, M):
    mx = gpu
    gen = torch.Generator().manual_seed(3)
    R, Y = torch.randn(M, 776, generator=gen).cuda(), torch.randn(M, 776, generator=gen).half().cuda()
    n = mx.Norm(LAYER, _vec(gen, 776), _vec(gen, 776))
    good = mx.muxq_residual_norm(R, Y, n, post=n)
    R[4, 100] = value
    got = mx.muxq_residual_norm(R, Y, n, post=n)
    keep = [i for i in range(M) if i != 4]
    for a, b in zip(good, got):
        assert torch.equal(a[keep], b[keep])


@pytest.mark.gpu
def test_results_that_are_not_wanted(gpu):
    mx = gpu
    gen = torch.Generator().manual_seed(4)
    R, Y = torch.randn(33, 264, generator=gen).cuda(), torch.randn(33, 264, generator=gen).half().cuda()
    n = mx.Norm(RMS, _vec(gen, 264))
    h, x = mx.muxq_residual_norm(R, Y, n, scale=0.5)
    h1, none = mx.muxq_residual_norm(R, Y, n, scale=0.5, want_x=False)
    none2, x2 = mx.muxq_residual_norm(R, Y, n, scale=0.5, want_h=False)
    assert none is None and none2 is None and torch.equal(h, h1) and torch.equal(x, x2)
    assert mx.muxq_residual_norm(R, None, n)[0] is None
    with pytest.raises(mx.MuxqError):
        mx.muxq_residual_norm(R, None, n, gate=_vec(gen, 264))


@pytest.mark.gpu
def test_columns_of_one_wider_matrix(gpu):
    """Y and X side by side in one matrix, as slices of a projection's result and the next one's input may be."""
    mx = gpu
    gen = torch.Generator().manual_seed(5)
    both = torch.randn(70, 2 * 264, generator=gen).half().cuda()
    R, n = torch.randn(70, 264, generator=gen).cuda(), mx.Norm(LAYER, _vec(gen, 264), _vec(gen, 264))
    want = mx.muxq_residual_norm(R, both[:, :264].clone(), n)
    Y = both[:, :264].clone()
    h, x = mx.muxq_residual_norm(R, both[:, :264], n, X=both[:, 264:])
    assert torch.equal(h, want[0]) and torch.equal(x, want[1]) and torch.equal(both[:, :264], Y)
    with pytest.raises(mx.MuxqError):
        mx.muxq_residual_norm(R, both[:, :264], n, X=both[:, 256:520])


@pytest.mark.gpu
def test_streams_and_graphs(gpu):
    """On another stream than the current one's default, captured, and replayed with new values in the same buffers."""
    mx = gpu
    gen = torch.Generator().manual_seed(6)
    n = mx.Norm(LAYER, _vec(gen, 1280), _vec(gen, 1280))
    R, Y = torch.randn(16, 1280, generator=gen).cuda(), torch.randn(16, 1280, generator=gen).half().cuda()
    H, X = torch.empty_like(R), torch.empty_like(Y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = mx.muxq_residual_norm(R, Y, n, post=n)
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            mx.muxq_residual_norm(R, Y, n, post=n, H=H, X=X)
            mx.muxq_residual_norm(H, Y, n, post=n, H=H, X=X)  # twice in a row, the stream in place
    torch.cuda.synchronize()
    for k in range(3):
        R.copy_(torch.randn(16, 1280, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        h, _ = mx.muxq_residual_norm(R, Y, n, post=n)
        h, x = mx.muxq_residual_norm(h, Y, n, post=n)
        assert torch.equal(h, H) and torch.equal(x, X)
    assert a[0].shape == R.shape


@pytest.mark.gpu
def test_offsets_beyond_32_bits(gpu):
    """Three rows a gigabyte of elements apart."""
    mx = gpu
    pitch = 1 << 30
    gen = torch.Generator().manual_seed(8)
    whole = torch.empty(2 * pitch + 64, dtype=torch.float16, device="cuda")
    R = whole.as_strided((3, 64), (pitch, 1))
    R.copy_(torch.randn(3, 64, generator=gen))
    n = mx.Norm(RMS)
    want = mx.muxq_residual_norm(R.contiguous(), None, n)[1]
    assert torch.equal(mx.muxq_residual_norm(R, None, n)[1], want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("M,D", [(5, 64), (5, 768), (700, 768), (700, 1280), (5, 5120), (600, 5120), (3, 16384), (600, 16384)])
def test_up_to_the_largest_values(gpu, M, D, kind):
    """Rows of values up to 1e18, whose squares add up to more than fp32 holds (D x 1e36), as the stream and as a block's result under post; the mean
    is near zero, or all but a few values are at the other end, 2e18 from them.  (What keeps the sum within fp32 is a power of two and rounds nothing.)"""
    mx = gpu
    gen = torch.Generator().manual_seed(M + D)
    v = (torch.rand(M, D, generator=gen) * 1.5 + 0.5) * 0.49e18 * (torch.randint(0, 2, (M, D), generator=gen) * 2.0 - 1.0)
    v[1] = -0.99e18
    v[1, :3] = 0.99e18
    v[2] = 0.99e18 * (torch.arange(D) % 2 * 2.0 - 1.0)
    v = v.cuda()
    n = mx.Norm(kind, _vec(gen, D), _vec(gen, D, 0.0), 1e-5)
    _, _, x, ex = reference(v, None, n, None, None, 1, 1.0)
    check(mx.muxq_residual_norm(v, None, n)[1], torch.float16, x, ex, "x")
    h, e, _, _ = reference(None, v, None, n, None, 1, 1.0)
    check(mx.muxq_residual_norm(None, v, None, post=n, want_x=False)[0], torch.float32, h, e, "h")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("M,D", [(3, 768), (600, 768), (3, 16384)])
def test_a_small_eps_and_values_beside_it(gpu, M, D, kind):
    """Squares far below those of activations, and an eps that does not cover them."""
    mx = gpu
    gen = torch.Generator().manual_seed(D + M)
    v = (torch.randn(M, D, generator=gen) * 1e-15).cuda()
    n = mx.Norm(kind, _vec(gen, D), None, 1e-32)
    _, _, x, ex = reference(v, None, n, None, None, 1, 1.0)
    check(mx.muxq_residual_norm(v, None, n)[1], torch.float16, x, ex, "x")


@pytest.mark.gpu
@pytest.mark.parametrize("M,D", [(4, 264), (700, 776), (700, 1040), (40, 2560), (650, 5120), (600, 8192)])
@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("weight,bias", [(True, True), (True, False), (False, True), (False, False)])
def test_weight_and_bias_each_alone(gpu, M, D, kind, weight, bias):
    """On both sides of the block and for either norm, with few and many channels a thread."""
    mx = gpu
    gen = torch.Generator().manual_seed(3 * M + D)
    R, Y = torch.randn(M, D, generator=gen).cuda(), torch.randn(M, D, generator=gen).half().cuda()
    norm = lambda: mx.Norm(kind, _vec(gen, D) if weight else None, _vec(gen, D, 0.3) if bias else None, 1e-5)
    pre, post = norm(), norm()
    H, X = mx.muxq_residual_norm(R, Y, pre, post=post, scale=0.7)
    h, e, x, ex = reference(R, Y, pre, post, None, 1, 0.7)
    check(H, F32, h, e, "h")
    check(X, F16, x, ex, "x")


@pytest.mark.gpu
def test_a_gate_beside_the_result_in_one_wider_matrix(gpu):
    """The gate is a row, or every third row, of columns that lie beside X's."""
    mx = gpu
    gen = torch.Generator().manual_seed(9)
    whole = torch.randn(66, 2 * 264, generator=gen).half().cuda()
    R, Y = torch.randn(66, 264, generator=gen).cuda(), torch.randn(66, 264, generator=gen).half().cuda()
    n, X = mx.Norm(RMS, _vec(gen, 264)), whole[:, :264]
    right = whole[:, 264:].clone()
    for gate, group in ((whole[7, 264:], 1), (whole[::3, 264:], 3)):
        want = mx.muxq_residual_norm(R, Y, n, gate=gate.clone(), gate_group=group)
        h, x = mx.muxq_residual_norm(R, Y, n, gate=gate, gate_group=group, X=X)
        assert torch.equal(h, want[0]) and torch.equal(x, want[1]) and torch.equal(whole[:, 264:], right)
    with pytest.raises(mx.MuxqError):
        mx.muxq_residual_norm(R, Y, n, gate=whole[7, 256:520], X=X)
