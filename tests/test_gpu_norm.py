"""lst_norm_forward, lst_norm_backward and lst_scores_coded against oracle.norms and
oracle.answers: sums and codes bit for bit, values and gradients within their roundings."""
import numpy as np
import pytest
import torch

import paper_1412_7091_amd as lst
from oracle import answers, norms

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24
SHAPES = [(1, 1), (3, 7), (2, 16), (17, 128), (5, 129), (33, 200), (9, 256), (4, 257), (70, 500),
          (1, 512), (6, 513), (8, 1024), (3, 1025), (11, 2048), (2, 2049), (5, 4096)]


def _np(t):
    return t.detach().double().cpu().numpy()


def _least(dtype):  # half of the smallest step
    return 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134


def _inputs(rows, cols, dtype, n=4):
    g = torch.Generator("cuda").manual_seed(rows * 5000 + cols)
    w = torch.randn(cols, device="cuda", generator=g) + 1
    scale = torch.exp2(torch.randint(-4, 5, (rows, 1), device="cuda", generator=g).float())
    return w, [(torch.randn((rows, cols), device="cuda", generator=g) * scale).to(dtype)
               for _ in range(n)]


def _check_forward(y, s, rstd, w, eps, dtype):
    want, q = norms.norm(_np(s), _np(w), eps)
    # the factor is rounded once, then two products
    off = 3.01 * U * np.abs(want)
    off = off + torch.finfo(dtype).eps / 2 * (np.abs(want) + off) + _least(dtype)
    assert (np.abs(_np(y) - want) <= off).all()
    if rstd is not None:
        assert (np.abs(_np(rstd) - q) <= 1.01 * U * q).all()


def _check_backward(got, s, w, eps, gy, gs):
    dx, dw = got
    S, W, G = _np(s), _np(w), _np(gy)
    want, want_w = norms.norm_grad(S, W, eps, G, None if gs is None else _np(gs))
    rows, cols = S.shape
    q = norms.norm(S, W, eps)[1][:, None]
    hat, a = np.abs(S * q), np.abs(G * W)
    mean = (a * hat).mean(axis=1, keepdims=True)
    # hat carries two roundings and a one; each term of the inner sum goes through at most 16
    # sums in its lane, 8 over the lanes and the division; then hat times that, the difference,
    # the factor (rounded once itself) and the sum with grad_sum
    off = U * q * (4 * a + hat * mean * (3 + 1 + 16 + 8 + 1 + 6)) * 1.01 + U * np.abs(want)
    off = off + torch.finfo(s.dtype).eps / 2 * (np.abs(want) + off) + _least(s.dtype)
    assert (np.abs(_np(dx) - want) <= off).all()
    # terms of two roundings of hat and a fused sum: those of a wave's rows, of the waves and of
    # the blocks
    off = U * (np.abs(G) * hat).sum(axis=0) * (3 + rows / 256 + 8 + 6 + 32 + 16) * 1.01
    assert (np.abs(_np(dw) - want_w) <= off).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_both_directions(gpu_lib, dtype, rows, cols):
    w, (x, r, gy, gs) = _inputs(rows, cols, dtype)
    layer = lst.RMSNorm(w, eps=1e-5)
    for res, more in ((None, None), (r, gs), (r, None)):
        y, s, rstd = layer.forward(x, res, save=True)
        if res is None:
            assert s is x
        else:
            assert torch.equal(s, (x.float() + r.float()).to(dtype))
        _check_forward(y, s, rstd, w, 1e-5, dtype)
        _check_backward(layer.backward(s, rstd, gy, more), s, w, 1e-5, gy, more)


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [24, 500, 1030])
def test_many_rows(gpu_lib, cols):
    """More rows than the backward pass has waves, and a number that no block divides."""
    w, (x, r, gy, gs) = _inputs(20_011, cols, torch.bfloat16)
    layer = lst.RMSNorm(w)
    y, s, rstd = layer.forward(x, r, save=True)
    _check_forward(y, s, rstd, w, 1e-6, torch.bfloat16)
    first = layer.backward(s, rstd, gy, gs)
    _check_backward(first, s, w, 1e-6, gy, gs)
    again = layer.backward(s, rstd, gy, gs)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [((1 << 24) + 37, 5), ((1 << 20) + 5, 1030)])
def test_more_rows_than_a_launch_has_blocks(gpu_lib, rows, cols):
    """2^20 blocks of 16 rows, or of one: rows of the second turn, and around its begin, are those
    of a call for them alone."""
    g = torch.Generator("cuda").manual_seed(cols)
    x = torch.randn((rows, cols), device="cuda", generator=g, dtype=torch.bfloat16)
    w = torch.randn(cols, device="cuda", generator=g) + 1
    layer = lst.RMSNorm(w)
    some = slice(rows - 300, rows)
    y, _, rstd = layer.forward(x, save=True)
    want = layer.forward(x[some], save=True)
    _check_forward(want[0], x[some], want[2], w, 1e-6, torch.bfloat16)
    assert torch.equal(y[some], want[0]) and torch.equal(rstd[some], want[2])
    assert torch.equal(y[:300], layer.forward(x[:300])[0])
    del y
    codes, scales, _ = layer.forward_coded(x)
    want = layer.forward_coded(x[some])
    assert torch.equal(codes[some], want[0]) and torch.equal(scales[some], want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_codes(gpu_lib, dtype, rows, cols):
    w, (x, r, _, _) = _inputs(rows, cols, dtype)
    layer = lst.RMSNorm(w)
    codes, scales, s = layer.forward_coded(x, r)
    assert torch.equal(s, (x.float() + r.float()).to(dtype))
    # y is computed in float64 and rounded to float32 before it is quantised
    want = answers.quantize(norms.norm(_np(s), _np(w), 1e-6)[0].astype(np.float32))
    assert np.array_equal(codes.cpu().numpy(), want[0])
    assert np.array_equal(scales.cpu().numpy(), want[1])


@pytest.mark.gpu
def test_codes_and_rows_in_one_call(gpu_lib):
    """The C entry gives both; the rows are those of a call without codes."""
    w, (x, r, _, _) = _inputs(13, 300, torch.bfloat16)
    layer = lst.RMSNorm(w)
    y, s, _ = layer.forward(x, r)
    codes, scales, _ = layer.forward_coded(x, r)
    y2, c2, s2 = torch.empty_like(y), torch.empty_like(codes), torch.empty_like(scales)
    code = lst.load_library().lst_norm_forward(
        lst.LST_BF16, 13, 300, x.data_ptr(), 300, r.data_ptr(), 300, w.data_ptr(), 1e-6, None, 0,
        y2.data_ptr(), 300, c2.data_ptr(), s2.data_ptr(), None,
        torch.cuda.current_stream().cuda_stream)
    assert code == lst.LST_OK
    assert torch.equal(y, y2) and torch.equal(codes, c2) and torch.equal(scales, s2)


@pytest.mark.gpu
@pytest.mark.parametrize("m,D,d", [(1, 33, 5), (7, 300, 129), (16, 257, 500), (17, 100, 300),
                                   (130, 515, 1024), (3, 40, 4096)])
def test_scores_of_coded_rows(gpu_lib, m, D, d):
    """Outputs for rows that came as codes are those for the rows, bit for bit; behind the norm
    they are those that the oracle has for its codes."""
    w, (x, _, _, _) = _inputs(m, d, torch.bfloat16)
    W = torch.randn((D, d), device="cuda", generator=torch.Generator("cuda").manual_seed(d))
    held = lst.EightBitOutputLayer(W)
    for dtype in (torch.float32, torch.bfloat16):
        assert torch.equal(held.scores(lst.lst_quantize(x), dtype=dtype),
                           held.scores(x, dtype=dtype))
    codes, scales, _ = lst.RMSNorm(w).forward_coded(x)
    got = held.scores((codes, scales))
    assert got.dtype == torch.float32
    want, bar = answers.scores(answers.values(codes.cpu().numpy(), scales.cpu().numpy()),
                               answers.values(held.codes.cpu().numpy(), held.scales.cpu().numpy()))
    assert (np.abs(_np(got) - want) <= bar + U * (np.abs(want) + bar)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [21, 520, 1500])
def test_strides_in_place_and_what_is_beside(gpu_lib, dtype, cols):
    rows = 9
    w, (a, b, c, e) = _inputs(rows, cols, dtype)
    layer = lst.RMSNorm(w)
    y, s, rstd = layer.forward(a, b, save=True)
    dx, dw = layer.backward(s, rstd, c, e)

    def held(*parts):  # the matrices as columns of one, between others
        whole = torch.randn((rows, len(parts) * (cols + 1) + 2), device="cuda").to(dtype)
        views = [whole[:, 1 + i * (cols + 1):][:, :cols] for i in range(len(parts))]
        for v, p in zip(views, parts):
            v.copy_(p)
        beside = torch.ones(whole.shape[1], dtype=torch.bool)
        for i in range(len(parts)):
            beside[1 + i * (cols + 1):1 + i * (cols + 1) + cols] = False
        return whole, views, beside, whole[:, beside].clone()

    whole, (x, r), beside, was = held(a, b)
    got = layer.forward(x, r, out=x, sum_out=r)
    assert got[0].data_ptr() == x.data_ptr() and got[1].data_ptr() == r.data_ptr()
    assert torch.equal(x, y) and torch.equal(r, s) and torch.equal(whole[:, beside], was)
    # the sum where x was, and a copy of x where there is nothing to add
    whole, (x, r), beside, was = held(a, b)
    got = layer.forward(x, r, sum_out=x)
    assert torch.equal(got[0], y) and got[1] is x and torch.equal(x, s) and torch.equal(r, b)
    got = layer.forward(a, sum_out=r)
    assert got[1] is r and torch.equal(r, a)
    codes, scales, _ = layer.forward_coded(a, b)
    x.copy_(a)
    r.copy_(b)
    got = layer.forward_coded(x, r, sum_out=r)
    assert torch.equal(r, s) and torch.equal(got[0], codes) and torch.equal(got[1], scales)
    assert torch.equal(whole[:, beside], was)
    for which in range(3):
        whole, views, beside, was = held(s, c, e)
        g, gw = layer.backward(views[0], rstd, views[1], views[2], out=views[which])
        assert torch.equal(g, dx) and torch.equal(gw, dw)
        assert torch.equal(whole[:, beside], was)
        assert all(torch.equal(v, p) for i, (v, p) in enumerate(zip(views, (s, c, e)))
                   if i != which)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 5), (9, 300), (3, 2049)])
def test_in_place_without_a_residual(gpu_lib, dtype, rows, cols):
    """y where x was: the sum that the backward pass reads is x as it was, and none is returned
    where there is none."""
    w, (x, _, gy, gs) = _inputs(rows, cols, dtype)
    layer = lst.RMSNorm(w)
    want, s, rstd = layer.forward(x, save=True)
    grads = layer.backward(s, rstd, gy, gs)
    a = x.clone()
    y, kept, rstd = layer.forward(a, out=a, save=True)
    assert y is a and torch.equal(a, want) and torch.equal(kept, x)
    for g, h in zip(layer.backward(kept, rstd, gy, gs), grads):
        assert torch.equal(g, h)
    a, b = x.clone(), torch.empty_like(x)
    y, kept, _ = layer.forward(a, out=a)
    assert torch.equal(y, want) and kept is None
    with pytest.raises(TypeError):
        layer.backward(kept, rstd, gy)
    a.copy_(x)
    y, kept, _ = layer.forward(a, out=a, sum_out=b)
    assert torch.equal(y, want) and kept is b and torch.equal(b, x)
    a = x.clone()
    assert lst.lst_norm_forward(a, w, out=a, rstd=rstd)[1].data_ptr() != a.data_ptr()
    none = x[:0]
    assert layer.forward(none, out=none)[1] is none


@pytest.mark.gpu
def test_extremes(gpu_lib):
    """Squares beyond float32's range, rows of zeros, tiny rows, infinities and no numbers."""
    w = torch.ones(40, device="cuda")
    x = torch.randn((8, 40), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    x[0] *= 2.0 ** 120
    x[1] = 3.0e38
    x[2] = 0
    x[3] *= 2.0 ** -60
    x[4, 3] = float("inf")
    x[5, 3] = float("nan")
    layer = lst.RMSNorm(w, eps=2.0 ** -100)
    y, s, rstd = layer.forward(x, save=True)
    fine = [0, 1, 2, 3, 6, 7]
    _check_forward(y[fine], x[fine], None, w, 2.0 ** -100, torch.float32)
    assert (y[2] == 0).all() and torch.isnan(y[5]).all()
    assert torch.isnan(y[4, 3]) and (y[4, :3] == 0).all() and rstd[4] == 0
    codes, scales, _ = layer.forward_coded(x)
    want = answers.quantize(norms.norm(_np(x), _np(w), 2.0 ** -100)[0].astype(np.float32))
    have = codes.cpu().numpy()
    nan = (want[0] & 127) == 127
    assert np.array_equal((have & 127) == 127, nan) and np.array_equal(have[~nan], want[0][~nan])
    assert np.array_equal(scales.cpu().numpy(), want[1])


@pytest.mark.gpu
def test_gradients_against_differences(gpu_lib):
    w, (x, r, gy, gs) = _inputs(19, 70, torch.float32)
    layer = lst.RMSNorm(w, eps=0.01)
    _, s, rstd = layer.forward(x, r, save=True)
    dx, dw = layer.backward(s, rstd, gy, gs)
    S, W = _np(s), _np(w)
    total = lambda S, W: (norms.norm(S, W, 0.01)[0] * _np(gy)).sum() + (S * _np(gs)).sum()  # noqa: E731
    rng = np.random.default_rng(1)
    for _ in range(3):
        u, v, h = rng.standard_normal(S.shape), rng.standard_normal(W.shape), 1e-6
        slope = (total(S + h * u, W) - total(S - h * u, W)) / (2 * h)
        assert abs(slope - (_np(dx) * u).sum()) < 1e-5 * np.linalg.norm(_np(dx)) * np.linalg.norm(u)
        slope = (total(S, W + h * v) - total(S, W - h * v)) / (2 * h)
        assert abs(slope - (_np(dw) * v).sum()) < 1e-5 * np.linalg.norm(_np(dw)) * np.linalg.norm(v)


@pytest.mark.gpu
def test_no_rows_and_streams(gpu_lib):
    w, (x, r, gy, _) = _inputs(300, 500, torch.bfloat16)
    layer = lst.RMSNorm(w)
    y, s, rstd = layer.forward(x[:0], save=True)
    assert y.shape == (0, 500) and rstd.shape == (0,)
    dx, dw = layer.backward(s, rstd, gy[:0])
    assert dx.shape == (0, 500) and (dw == 0).all()
    want = layer.forward(x, r, save=True)
    grads = layer.backward(want[1], want[2], gy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer.forward(x, r, save=True)
        got_grads = layer.backward(got[1], got[2], gy)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((*want, *grads), (*got, *got_grads)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_captured(gpu_lib):
    w, (x, r, gy, gs) = _inputs(257, 300, torch.float16)
    layer = lst.RMSNorm(w)
    layer.backward(*layer.forward(x, r, save=True)[1:], gy, gs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, s, rstd = layer.forward(x, r, save=True)
        dx, dw = layer.backward(s, rstd, gy, gs)
        codes, scales, _ = layer.forward_coded(x, r)
    for i in range(4):
        x.copy_(torch.randn_like(x) * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, s, rstd, dx, dw, codes, scales)]
        e = layer.forward(x, r, save=True)
        want = [*e, *layer.backward(e[1], e[2], gy, gs), *layer.forward_coded(x, r)[:2]]
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals_on_the_host():
    lib, ok, bad = lst.load_library(), lst.LST_OK, lst.LST_EINVAL
    p = 4096  # never read: every call is refused, or has no rows

    def forward(dtype=0, rows=2, cols=8, x=p, ldx=8, r=None, ldr=0, w=p, eps=1e-6, s=None, lds=8,
                y=p, ldy=8, codes=None, scales=None):
        return lib.lst_norm_forward(dtype, rows, cols, x, ldx, r, ldr, w, eps, s, lds, y, ldy,
                                    codes, scales, None, None)

    assert forward(rows=0) == ok
    for kw in (dict(dtype=3), dict(rows=-1), dict(rows=(1 << 40) + 1), dict(cols=0),
               dict(cols=4097), dict(x=None), dict(ldx=7), dict(r=p, ldr=7), dict(w=None),
               dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(s=p + 4, lds=7),
               dict(ldy=9), dict(s=p, lds=9, y=p + 4), dict(r=p + 4, ldr=9, y=p + 4),
               dict(y=None), dict(ldy=7), dict(s=p, y=p), dict(codes=p), dict(scales=p),
               dict(codes=p + 8, scales=p)):
        assert forward(**kw) == bad, kw

    def backward(dtype=0, rows=2, cols=8, s=p, lds=8, w=p, q=p, gy=p, ldgy=8, gs=None, ldgs=0,
                 gx=p, ldgx=8, gw=p, work=p):
        return lib.lst_norm_backward(dtype, rows, cols, s, lds, w, q, gy, ldgy, gs, ldgs, gx, ldgx,
                                     gw, work, None)

    for kw in (dict(dtype=-1), dict(rows=-1), dict(cols=0), dict(cols=4097), dict(s=None),
               dict(lds=7), dict(w=None), dict(q=None), dict(gy=None), dict(ldgy=7),
               dict(ldgx=9), dict(gy=p + 4, ldgy=9, gx=p + 4), dict(gs=p + 4, ldgs=9, gx=p + 4),
               dict(gs=p, ldgs=7), dict(gx=None), dict(ldgx=7), dict(gw=None), dict(work=None),
               dict(work=p + 4)):
        assert backward(**kw) == bad, kw
    assert lib.lst_norm_workspace(-1, 8) == -1 and lib.lst_norm_workspace(1, 4097) == -1
    assert lib.lst_norm_workspace(1 << 30, 512) == 512 * 512 * 4
    coded = lambda m=2, d=8, h=p, hs=p, c=p, o=p, ldo=9, work=p, out=0: lib.lst_scores_coded(  # noqa: E731
        out, m, 9, d, h, hs, c, p, o, ldo, work, None)
    assert coded(m=0) == ok
    for kw in (dict(m=-1), dict(d=0), dict(h=None), dict(hs=None), dict(h=p + 8), dict(c=p + 8),
               dict(o=None), dict(ldo=8), dict(work=None), dict(out=7)):
        assert coded(**kw) == bad, kw


def test_tensors_on_the_host_and_shapes_are_refused():
    with pytest.raises(TypeError):
        lst.lst_norm_forward(torch.zeros(2, 3), torch.ones(3))
    with pytest.raises((TypeError, ValueError)):
        lst.lst_scores_coded(*(torch.zeros((2, 128), dtype=torch.uint8),) * 4)
    with pytest.raises(ValueError):
        lst.RMSNorm(torch.ones(2, 3))


@pytest.mark.gpu
def test_refusals_of_tensors(gpu_lib):
    x, w = torch.zeros((4, 6), device="cuda"), torch.ones(6, device="cuda")
    layer = lst.RMSNorm(w)
    for bad in (lambda: lst.RMSNorm(w.bfloat16()), lambda: layer.forward(x.double()),
                lambda: layer.forward(x[:, :5]), lambda: layer.forward(x, x.bfloat16()),
                lambda: layer.forward(x, x[:3]), lambda: layer.forward(x.t()),
                lambda: layer.forward(x, out=x.new_empty((4, 5))),
                lambda: layer.backward(x, w[:3], x), lambda: layer.backward(x, None, x)):
        with pytest.raises((TypeError, ValueError, lst.LstError)):
            bad()
    held = lst.EightBitOutputLayer(torch.zeros((9, 200), device="cuda"))
    codes, scales = lst.lst_quantize(x)
    with pytest.raises(ValueError):
        held.scores((codes, scales))
