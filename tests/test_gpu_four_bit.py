"""lst_quantize_four and lst_scores_four against oracle.answers: codes and scales bit for bit,
outputs within the roundings of a float32 sum."""
import numpy as np
import pytest
import torch

import paper_1412_7091_amd as lst
from oracle import answers

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _np(t):
    return t.detach().double().cpu().numpy()


def _check_codes(x, got):
    codes, scales = answers.quantize_four(_np(x))
    assert np.array_equal(got[1].cpu().numpy(), scales)
    # what a block without a number holds beside its values that are not finite is not said
    keep = np.repeat(scales != 255, 16, axis=1)
    assert np.array_equal(got[0].cpu().numpy()[keep], codes[keep])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (5, 32), (2, 33), (33, 500), (7, 1024),
                                       (2, 4096), (65, 15)])
def test_quantize(gpu_lib, dtype, rows, cols):
    g = torch.Generator("cuda").manual_seed(rows + 10 * cols)
    x = torch.randn((rows, cols), device="cuda", generator=g).to(dtype)
    _check_codes(x, lst.lst_quantize_four(x))
    big = torch.zeros((rows, cols + 5), device="cuda", dtype=dtype)
    big[:, 1:1 + cols] = x
    a, b = lst.lst_quantize_four(x), lst.lst_quantize_four(big[:, 1:1 + cols])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.gpu
def test_quantize_borders(gpu_lib):
    """Largest values at and beside the borders of the scale; ties and values beside them; zeros
    and their signs; extremes; not finite."""
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn((28, 96), device="cuda", generator=g)
    for i, v in enumerate((6.0, 7.0, 1.5, 3.0, 2.0 ** -100, 2.0 ** 100, 0.75)):
        at = torch.full((1,), v, device="cuda")
        x[3 * i] = x[3 * i].clamp(-1, 1) * v * 0.99
        x[3 * i + 1], x[3 * i + 2] = x[3 * i], x[3 * i]
        x[3 * i, 5] = v
        x[3 * i + 1, 5] = torch.nextafter(at, 2 * at)
        x[3 * i + 2, 5] = -torch.nextafter(at, 0 * at)
    x[21] = 0
    x[22, :32], x[22, 32:64], x[22, 64:] = 1e-41, 3.4e38, -0.0
    x[23, 7], x[23, 40], x[23, 69] = float("inf"), -float("inf"), float("nan")
    x[24] = torch.randn(96, device="cuda", generator=g) * 2.0 ** -127
    up = torch.from_numpy(answers.E2M1).cuda().float()
    t = torch.cat((up, (up[1:] + up[:-1]) / 2))
    t = torch.cat((t, torch.nextafter(t[8:], t[8:] * 2), torch.nextafter(t[8:], t[8:] * 0)))
    x[25], x[26] = 0, 0
    for row, sign in ((25, 1.0), (26, -1.0)):
        x[row, 1:1 + 15], x[row, 33:33 + 14] = sign * t[:15], sign * t[15:]
        x[row, 0::32] = 6.0  # the scale is one in every block
    _check_codes(x, lst.lst_quantize_four(x))


def _check_scores(H, layer, got):
    hq = answers.values_four(*answers.quantize_four(_np(H)))
    want, bar = answers.scores(hq, answers.values_four(layer.codes.cpu().numpy(),
                                                       layer.scales.cpu().numpy()))
    bar = bar + torch.finfo(got.dtype).eps / 2 * (np.abs(want) + bar)
    if got.dtype == torch.float16:
        bar += 2.0 ** -25
    assert (np.abs(_np(got) - want) <= bar).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m,D,d", [
    (1, 1, 1), (1, 15, 32), (2, 16, 33), (5, 63, 500), (16, 64, 37), (17, 65, 300),
    (33, 1000, 500), (64, 127, 512), (65, 128, 1024), (100, 129, 130), (128, 2001, 500),
    (129, 257, 256), (300, 700, 385), (513, 4097, 128), (3, 300, 4096), (40, 270, 4096),
    (130, 300, 1153), (16, 8200, 700), (20, 60, 16),
    # parts of H's rows that LDS just holds, and one tile more
    (256, 200, 1000), (272, 200, 1000), (513, 300, 1000), (528, 70, 1024), (1100, 90, 600),
    (1850, 50, 120), (1841, 33, 100)])
def test_scores(gpu_lib, m, D, d):
    g = torch.Generator("cuda").manual_seed(m + D + d)
    W = torch.randn((D, d), device="cuda", generator=g) / d ** 0.5
    H = torch.randn((m, d), device="cuda", generator=g)
    # rows and blocks of very different sizes
    W *= torch.exp2(torch.randint(-9, 9, (D, 1), device="cuda", generator=g).float())
    W[:, :d // 2] *= 4096
    layer = lst.FourBitOutputLayer(W)
    got = layer.scores(H)
    assert got.dtype == torch.float32 and got.shape == (m, D)
    _check_scores(H, layer, got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("m", [1, 20, 60, 140])
def test_scores_types(gpu_lib, dtype, out, m):
    g = torch.Generator("cuda").manual_seed(m)
    W = torch.randn((333, 200), device="cuda", generator=g)
    H = torch.randn((m, 200), device="cuda", generator=g).to(dtype)
    layer = lst.FourBitOutputLayer(W)
    _check_scores(H, layer, layer.scores(H, dtype=out))


@pytest.mark.gpu
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("m", [6, 37])
def test_scores_strides_and_what_is_beside(gpu_lib, out, m):
    D, d = 203, 150
    g = torch.Generator("cuda").manual_seed(12)
    W = torch.randn((D, d), device="cuda", generator=g)
    big = torch.randn((m, d + 9), device="cuda", generator=g)
    whole = torch.full((m + 2, D + 7), 5.0, device="cuda", dtype=out)
    layer = lst.FourBitOutputLayer(W)
    view = whole[1:1 + m, 3:3 + D]
    got = layer.scores(big[:, 3:3 + d], out=view)
    assert got.data_ptr() == view.data_ptr()
    _check_scores(big[:, 3:3 + d], layer, view)
    whole[1:1 + m, 3:3 + D] = 5.0
    assert (whole == 5.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("out", TYPES)
def test_rows_of_new_outputs_begin_at_lines(gpu_lib, out):
    g = torch.Generator("cuda").manual_seed(2)
    layer = lst.FourBitOutputLayer(torch.randn((203, 40), device="cuda", generator=g))
    H = torch.randn((33, 40), device="cuda", generator=g)
    got = layer.scores(H, dtype=out)
    assert got.shape == (33, 203) and got.stride(1) == 1
    assert got.stride(0) * got.element_size() == -(-203 * got.element_size() // 128) * 128
    tight = torch.empty((33, 203), device="cuda", dtype=out)
    assert torch.equal(layer.scores(H, out=tight), got)
    assert layer.scores(H[:1]).is_contiguous()
    assert lst.FourBitOutputLayer(torch.ones((256, 40), device="cuda")).scores(H).is_contiguous()


@pytest.mark.gpu
@pytest.mark.parametrize("out", TYPES[:2])
@pytest.mark.parametrize("m,D,d,step", [
    # up to 16 rows of H: 65 536 rows of W a round of waves, with and without words of exponents
    (1, 140_001, 300, 65_536), (16, 140_001, 512, 65_536), (3, 70_003, 1000, 65_536),
    (16, 131_073, 40, 65_536),
    # 131 072 a round, 65 536 above 512 columns; the third round reuses the first one's registers
    (17, 262_221, 33, 131_072), (40, 262_221, 300, 131_072), (33, 262_145, 450, 131_072),
    (20, 140_000, 512, 131_072), (30, 400_009, 100, 131_072),
    (18, 131_149, 700, 65_536), (20, 131_149, 1024, 65_536), (17, 131_073, 520, 65_536),
    (40, 70_000, 1000, 65_536), (17, 300_001, 896, 65_536),
    # several parts of H: 10 blocks of a part on an XCD
    (528, 50_001, 1024, 20_480), (257, 66_000, 1000, 32_768)])
def test_scores_of_many_rows_of_weights(gpu_lib, m, D, d, step, out):
    """More rows of W than all waves take at once: rows around the end of each round against the
    oracle, all of them against calls for parts of W, which one round takes, and what is beside."""
    g = torch.Generator("cuda").manual_seed(m + D + d)
    W = torch.randn((D, d), device="cuda", generator=g) / d ** 0.5
    W *= torch.exp2(torch.randint(-9, 9, (D, 1), device="cuda", generator=g).float())
    H = torch.randn((m, d), device="cuda", generator=g)
    layer = lst.FourBitOutputLayer(W)
    got = layer.scores(H, dtype=out)
    near = [np.arange(r - 70, r + 70) for r in range(0, D + step, step)] + [np.arange(D - 70, D)]
    rows = np.unique(np.concatenate(near))
    rows = torch.from_numpy(rows[(rows >= 0) & (rows < D)]).cuda()
    part = lst.FourBitOutputLayer(W[:1])
    part.codes, part.scales = layer.codes[rows], layer.scales[rows]
    _check_scores(H, part, got[:, rows])
    for a in range(0, D, 8000):
        some = slice(a, a + 8000)
        want = lst.lst_scores_four(H, layer.codes[some], layer.scales[some], dtype=out)
        assert torch.equal(got[:, some], want), a
    for wide, at in ((D, 0), (D + 7, 3)):
        whole = torch.full((m + 2, wide), 5.0, device="cuda", dtype=out)
        view = whole[1:1 + m, at:at + D]
        assert torch.equal(layer.scores(H, out=view), got)
        view.fill_(5.0)
        assert (whole == 5.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m", [3, 35])
def test_sums_of_sizes_far_apart(gpu_lib, m):
    """Blocks 2^20 apart that one instruction adds up: what float32 keeps of the smaller stays."""
    d = 256
    W = torch.zeros((40, d), device="cuda")
    H = torch.zeros((m, d), device="cuda")
    W[:, 0], H[:, 0] = 6.0 * 2.0 ** 10, 6.0 * 2.0 ** 8
    W[:, 32], H[:, 33] = 0.5, 0.5
    W[:, 33], H[:, 34] = 1.5, 3.0
    W[:, 200], H[:, 200] = 3.0, 0.5
    layer = lst.FourBitOutputLayer(W)
    got = layer.scores(H)
    assert (got == 36.0 * 2.0 ** 18 + 0.75 + 1.5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m", [2, 19])
def test_what_is_not_finite(gpu_lib, m):
    """A value that is not finite makes its row's outputs no numbers, and those alone."""
    g = torch.Generator("cuda").manual_seed(m)
    W = torch.randn((70, 300), device="cuda", generator=g)
    H = torch.randn((m, 300), device="cuda", generator=g)
    W[5, 290], W[40, 1], H[1, 100] = float("inf"), float("nan"), -float("inf")
    got = lst.FourBitOutputLayer(W).scores(H)
    nan = torch.zeros((m, 70), dtype=torch.bool, device="cuda")
    nan[:, 5], nan[:, 40], nan[1] = True, True, True
    assert torch.equal(torch.isnan(got), nan)


@pytest.mark.gpu
def test_extreme_scales(gpu_lib):
    W = torch.randn((20, 64), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    H = torch.randn((3, 64), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    W[:10] *= 2.0 ** 100
    W[10:] *= 2.0 ** -90
    for scale in (2.0 ** 20, 2.0 ** -20):
        layer = lst.FourBitOutputLayer(W)
        _check_scores(H * scale, layer, layer.scores(H * scale))
    W[:] = 0
    assert (lst.FourBitOutputLayer(W).scores(H) == 0).all()


@pytest.mark.gpu
def test_layer_load_sample_and_streams(gpu_lib):
    g = torch.Generator("cuda").manual_seed(8)
    W, V = (torch.randn((900, 64), device="cuda", generator=g) for _ in range(2))
    H = torch.randn((50, 64), device="cuda", generator=g)
    layer = lst.FourBitOutputLayer(lst.FactoredOutputLayer(W))
    at = layer.codes.data_ptr()
    assert torch.equal(layer.codes, lst.lst_quantize_four(W)[0])
    layer.load(V)
    assert layer.codes.data_ptr() == at
    want = layer.scores(H)
    _check_scores(H, layer, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer.scores(H)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(want, got)
    u = torch.rand(50, device="cuda", generator=g)
    tokens, _ = layer.sample(H, u)
    assert torch.equal(tokens, lst.lst_sample(want, u)[0])
    with pytest.raises(TypeError):
        layer.scores(lst.lst_quantize_four(H))
    with pytest.raises(ValueError):
        layer.scores(H[:, :60])
    assert layer.scores(H[:0]).shape == (0, 900)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [4, 90])
def test_captured(gpu_lib, m):
    g = torch.Generator("cuda").manual_seed(9)
    W = torch.randn((700, 130), device="cuda", generator=g)
    H = torch.randn((m, 130), device="cuda", generator=g)
    layer = lst.FourBitOutputLayer(W)
    layer.scores(H)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.load(W)
        O = layer.scores(H)
    for i in range(4):
        H.copy_(torch.randn((m, 130), device="cuda"))
        W.copy_(torch.randn((700, 130), device="cuda") * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone()
        assert torch.equal(got, lst.FourBitOutputLayer(W).scores(H))


def test_refusals_on_the_host():
    lib, ok, bad = lst.load_library(), lst.LST_OK, lst.LST_EINVAL
    p = 4096  # never read: every call is refused, or has no rows

    def quantize(dtype=0, rows=2, cols=8, x=p, ldx=8, codes=p, scales=p):
        return lib.lst_quantize_four(dtype, rows, cols, x, ldx, codes, scales, None)

    assert quantize(rows=0) == ok
    for kw in (dict(dtype=3), dict(rows=-1), dict(cols=0), dict(cols=4097), dict(x=None),
               dict(ldx=7), dict(codes=None), dict(codes=p + 8), dict(scales=None),
               dict(rows=(1 << 30) - 63), dict(rows=(1 << 23), cols=4096, ldx=4096)):
        assert quantize(**kw) == bad, kw

    def scores(dtype=0, out=0, m=2, D=9, d=8, H=p, ldh=8, codes=p, scales=p, O=p, ldo=9, work=p):
        return lib.lst_scores_four(dtype, out, m, D, d, H, ldh, codes, scales, O, ldo, work, None)

    assert scores(m=0) == ok
    for kw in (dict(dtype=3), dict(out=3), dict(m=-1), dict(D=0), dict(d=0), dict(d=4097),
               dict(H=None), dict(ldh=7), dict(codes=None), dict(codes=p + 8), dict(scales=None),
               dict(O=None), dict(ldo=8), dict(work=None), dict(work=p + 8),
               dict(m=(1 << 20) + 1), dict(D=(1 << 36) + 1, ldo=1 << 37),
               dict(m=17, D=1 << 33, ldo=1 << 33)):
        assert scores(**kw) == bad, kw
    assert lib.lst_scores_four_workspace(-1, 8) == -1
    assert lib.lst_scores_four_workspace(1, 4097) == -1
    assert lib.lst_scores_four_workspace(17, 129) == 2 * 2 * 1024 + 2 * 256


def test_tensors_on_the_host_are_refused():
    with pytest.raises(TypeError):
        lst.lst_quantize_four(torch.zeros((2, 3)))
