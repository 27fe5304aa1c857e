"""lst_dropout against oracle.between: masks bit for bit, values within their roundings."""
import numpy as np
import pytest
import torch

import paper_1412_7091_amd as lst
from oracle import between

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _want(x, res, p, seed, offset):
    keep, factor = between.keep_mask(*x.shape, p, seed, offset)
    y = np.where(keep, x.double().cpu().numpy() * factor, 0.0)
    off = 2 * 2.0 ** -24 * np.abs(y)  # the rounded factor and the product
    if res is not None:
        y = y + res.double().cpu().numpy()
        off += 2.0 ** -24 * np.abs(y)
    return y, off + torch.finfo(x.dtype).eps / 2 * (np.abs(y) + off), keep


def _check(got, want, off):
    assert (np.abs(got.double().cpu().numpy() - want) <= off).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (2, 9), (16, 32), (7, 500),
                                       (130, 33), (1, 4097)])
def test_values(gpu_lib, dtype, rows, cols):
    g = torch.Generator("cuda").manual_seed(rows * 10_000 + cols)
    x, res = (torch.randn((rows, cols), device="cuda", generator=g).to(dtype) for _ in range(2))
    layer = lst.Dropout(0.3, seed=0xFEDCBA9876543210)
    for r in (None, res):
        want, off, _ = _want(x, r, 0.3, layer.seed, 1 << 33 | 5)
        _check(layer.forward(x, 1 << 33 | 5, residual=r), want, off)


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 1e-5, 0.5, 0.999, 1.0])
def test_probabilities(gpu_lib, p):
    x = torch.randn((9, 50), device="cuda")
    want, off, keep = _want(x, None, p, 1, 2)
    got = lst.lst_dropout(x, p, 1, 2)
    _check(got, want, off)
    assert ((got.cpu().numpy() != 0) == keep).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_in_place_and_what_is_beside(gpu_lib, dtype):
    rows, cols = 13, 21
    whole = torch.randn((rows, 2 * cols + 3), device="cuda").to(dtype)
    keep_whole = whole.clone()
    x, res = whole[:, 1:1 + cols], whole[:, 1 + cols:1 + 2 * cols]
    want, off, _ = _want(x, res, 0.4, 9, 8)
    got = lst.lst_dropout(x, 0.4, 9, 8, residual=res, out=res)
    assert got.data_ptr() == res.data_ptr()
    _check(res, want, off)
    beside = torch.ones(whole.shape[1], dtype=torch.bool)
    beside[1 + cols:1 + 2 * cols] = False
    assert torch.equal(whole[:, beside], keep_whole[:, beside])


@pytest.mark.gpu
def test_dropped_elements_are_zero_whatever_they_hold(gpu_lib):
    x = torch.full((4, 64), float("nan"), device="cuda")
    x[1], x[2] = float("inf"), -float("inf")
    y = lst.lst_dropout(x, 0.5, 3, 4).cpu().numpy()
    keep, _ = between.keep_mask(4, 64, 0.5, 3, 4)
    assert (y[~keep] == 0).all()
    assert np.isnan(y[0][keep[0]]).all() and (y[1][keep[1]] == np.inf).all()


@pytest.mark.gpu
def test_backward_has_the_forward_mask(gpu_lib):
    layer = lst.Dropout(0.35, seed=11)
    x, dy = (torch.rand((33, 70), device="cuda") + 1 for _ in range(2))
    y, dx = layer.forward(x, 6), layer.backward(dy, 6)
    assert torch.equal(y == 0, dx == 0)
    want, off, _ = _want(dy, None, 0.35, 11, 6)
    _check(dx, want, off)
    # the loss sum(y dy) is linear in x: its slope along v is sum(dx v)
    v = torch.randn_like(x)
    slope = ((layer.forward(x + v, 6).double() - layer.forward(x - v, 6).double()) / 2 *
             dy.double()).sum()
    assert abs(float(slope - (dx.double() * v.double()).sum())) < 33 * 70 * 16 * 2.0 ** -24


@pytest.mark.gpu
def test_replays_draw_new_masks(gpu_lib):
    x = torch.randn((40, 96), device="cuda")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        lst.lst_dropout(x, 0.5, 5, 100, counter=counter)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y = lst.lst_dropout(x, 0.5, 5, 100, counter=counter)
            counter += 1
    torch.cuda.synchronize()
    counter.zero_()
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, lst.lst_dropout(x, 0.5, 5, 100 + k))


@pytest.mark.gpu
def test_large_and_empty(gpu_lib):
    """Rows past 2^31 elements, against the same rows drawn by themselves."""
    assert lst.lst_dropout(torch.empty((0, 8), device="cuda"), 0.5, 1).shape == (0, 8)
    rows, cols = 70_000, 32_768
    x = torch.ones((rows, cols), device="cuda", dtype=torch.bfloat16)
    lst.lst_dropout(x, 0.5, 21, 22, out=x)
    for row in (0, 65_535, 65_536, rows - 1):
        words = [between.philox((c, row, 22, 0), (21, 0)) for c in (0, cols // 8 - 1)]
        bits = np.array([w >> s & 0xFFFF for block in words for w in block for s in (0, 16)])
        got = torch.cat((x[row, :8], x[row, -8:])).float().cpu().numpy()
        assert ((got == 2) == (bits >= 32_768)).all() and set(got) <= {0.0, 2.0}
    share = float((x != 0).sum(dtype=torch.int64)) / x.numel()
    assert abs(share - 0.5) < 1e-4  # nine standard deviations


@pytest.mark.gpu
def test_refusals(gpu_lib):
    x = torch.zeros((4, 8), device="cuda")
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises((lst.LstError, ValueError)):
            lst.lst_dropout(x, p, 1)
    with pytest.raises(ValueError):
        lst.lst_dropout(x, 0.5, -1)
    with pytest.raises(TypeError):
        lst.lst_dropout(x.double(), 0.5, 1)
    with pytest.raises(TypeError):
        lst.lst_dropout(x, 0.5, 1, residual=x.half())
    with pytest.raises(TypeError):
        lst.lst_dropout(x, 0.5, 1, out=x.cpu())
    with pytest.raises(ValueError):
        lst.lst_dropout(x.T, 0.5, 1)
    with pytest.raises(ValueError):
        lst.lst_dropout(x[:1].expand(4, 8), 0.5, 1)
    with pytest.raises(ValueError):
        lst.lst_dropout(x, 0.5, 1, residual=x[:2])


def test_refusals_on_host():
    lib = lst.load_library()
    P = 16  # never dereferenced

    def call(dtype=0, rows=2, cols=8, x=P, ldx=8, res=None, ldr=0, y=P, ldy=8, p=0.5):
        return lib.lst_dropout(dtype, rows, cols, x, ldx, res, ldr, y, ldy, p, 1, 0, None, None)

    bad = [dict(dtype=3), dict(rows=-1), dict(rows=(1 << 32) + 1), dict(cols=0), dict(x=None),
           dict(y=None), dict(ldx=7), dict(ldy=7), dict(res=P, ldr=7), dict(p=-1e-9),
           dict(p=1.5), dict(p=float("nan"))]
    for kw in bad:
        assert call(**kw) == lst.LST_EINVAL, kw
    assert call(rows=0, x=None, y=None) == lst.LST_OK
    with pytest.raises(ValueError):
        lst.Dropout(1.5)
    with pytest.raises(TypeError):
        lst.lst_dropout(torch.zeros(2, 8), 0.5, 1)


def test_sizes_behind_the_limits():
    """Refused on the host: columns counted in 32 bits with a block's step behind the last one,
    and launches of more than 2^32 threads."""
    lib = lst.load_library()
    P = 16  # never dereferenced

    def call(rows, cols):
        return lib.lst_dropout(1, rows, cols, P, cols, None, 0, P, cols, 0.5, 1, 0, None, None)

    for rows, cols in ((1, (1 << 30) + 1), (1, 0x7FFFFFFF), (1 << 32, 64)):
        assert call(rows, cols) == lst.LST_EINVAL, (rows, cols)
