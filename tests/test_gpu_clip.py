"""lst_clip against oracle.norms: the norm, and every element within its roundings."""
import ctypes
import time

import numpy as np
import pytest
import torch

import paper_1412_7091_amd as lst
from oracle import norms

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24


def _np(t):
    return t.detach().double().cpu().numpy()


def _check(before, after, norm, max_norm):
    """before, after: arrays in float64, after with its torch type."""
    n, f, want = norms.clip(before, max_norm)
    # sums in float64, whose own roundings are far below this one
    assert abs(float(norm) - n) <= 1.01 * U * n
    for w, a in zip(want, after):
        if f == 1.0:
            assert np.array_equal(_np(a), w)
            continue
        off = 2.01 * U * np.abs(w)  # the factor and the product
        off = off + torch.finfo(a.dtype).eps / 2 * (np.abs(w) + off)
        off += 2.0 ** -25 if a.dtype == torch.float16 else 2.0 ** -134
        assert (np.abs(_np(a) - w) <= off).all()


def _tensors(shapes, seed=0, kind=None):
    g = torch.Generator("cuda").manual_seed(seed)
    return [(torch.randn(s, device="cuda", generator=g) * 2.0 ** (i % 5 - 2)).to(
        kind or TYPES[i % 3]) for i, s in enumerate(shapes)]


SHAPES = [(1,), (7,), (3, 5), (1, 1), (8,), (500,), (500, 1000), (33, 129), (2, 3, 4), (), (0,),
          (4, 0), (8192,), (8193,), (130, 64), (1, 20_000)]


@pytest.mark.gpu
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("max_norm", [0.0, 1e-3, 500.0, 1e9, float("inf")])
def test_of_many_shapes_and_types(gpu_lib, apart, max_norm):
    tensors = _tensors(SHAPES)
    before = [_np(t) for t in tensors]
    out = [torch.full_like(t, 9.0) for t in tensors] if apart else None
    norm = lst.lst_clip(tensors, max_norm, out=out)
    assert norm.shape == ()
    _check(before, out or tensors, norm, max_norm)
    if apart:
        assert all(np.array_equal(_np(t), b) for t, b in zip(tensors, before))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 59, 60, 61, 200])
def test_numbers_of_tensors(gpu_lib, dtype, n):
    tensors = _tensors([(i % 37 + 1, i % 11 + 1) for i in range(n)], n, dtype)
    tensors.insert(n // 2, tensors[0].new_empty((0, 3)))
    before = [_np(t) for t in tensors]
    norm = lst.lst_clip(tensors, 2.0)
    _check(before, tensors, norm, 2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_columns_of_wider_matrices(gpu_lib, dtype):
    """Gradients that are columns of one matrix, and what is beside them."""
    whole = torch.randn((301, 80), device="cuda").to(dtype)
    a, b, c = whole[:, :33], whole[:, 33:50], whole[::2, 60:]
    was = whole.clone()
    before = [_np(t) for t in (a, b, c)]
    norm = lst.lst_clip([a, b], 3.0)
    _check(before[:2], [a, b], norm, 3.0)
    assert torch.equal(whole[:, 50:], was[:, 50:])
    target = torch.zeros((301, 90), device="cuda", dtype=dtype)
    norm = lst.lst_clip([c], 1.0, out=[target[:151, 3:23]])
    _check(before[2:], [target[:151, 3:23]], norm, 1.0)
    target[:151, 3:23] = 0
    assert (target == 0).all() and torch.equal(whole[:, 50:], was[:, 50:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_single_rows_beside_columns(gpu_lib, dtype):
    """A row, and a vector, whose memory lies between the rows of another matrix: taken where they
    share no element, on either side of it, and refused where they share one."""
    whole = torch.randn((100, 64), device="cuda").to(dtype)
    flat = whole.view(-1)
    for others in ((whole[:, :32], whole[3:4, 32:]), (whole[3:4, 32:], whole[:, :32]),
                   (whole[:, :32], whole[99, 32:], whole[0, 32:]),
                   (whole[1:, 8:40], flat[:72], flat[104:136], whole[99, 40:]),
                   (whole[5:6, 1:2], whole[5:, 2:], whole[:, :1])):
        before = [_np(t) for t in others]
        _check(before, others, lst.lst_clip(others, 1.5), 1.5)
    for others in ((whole[:, :33], whole[3:4, 32:]), (whole[3, 32:], whole[:, :33]),
                   (whole[1:, 8:40], flat[:73]), (whole[1:, 8:40], flat[103:136]),
                   (whole[:, 8:40], flat[104:137]), (whole[:, 8:40], flat[40:136])):
        with pytest.raises(lst.LstError):
            lst.lst_clip(others, 1.5)


@pytest.mark.gpu
def test_lists_within_one_matrix(gpu_lib):
    """Lists drawn from one piece of memory: those are refused in which an element that is written
    is in two (or whose rows of different strides reach into each other), and no others; of those
    that are taken every element is right."""
    rng = np.random.default_rng(7)
    taken = refused = 0
    for _ in range(400):
        memory = torch.randn(1200, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        used, lists, spans = np.zeros(1200, int), ([], []), []
        wide = rng.integers(8, 40, 2) if rng.random() < 0.3 else rng.integers(8, 40, 1).repeat(2)
        shared = False
        for _ in range(rng.integers(2, 6)):
            rows = int(rng.choice([1, 1, 2, 7, 20]))
            cols = int(rng.integers(1, 8 if rows > 1 else 60))
            apart = rng.random() < 0.3
            for k in range(2):
                ld = int(rng.choice(wide))
                at = int(rng.integers(0, 1200 - (rows - 1) * ld - cols + 1))
                if k and not apart:
                    lists[1].append(None)
                    continue
                view = torch.as_strided(memory, (rows, cols), (ld, 1), at)
                lists[k].append(view)
                place = (at + ld * np.arange(rows)[:, None] + np.arange(cols)).ravel()
                written = k == 1 or not apart
                shared |= bool((used[place] >= (1 if written else 2)).any())
                used[place] |= 2 if written else 1
                for s in spans if rows > 1 else ():
                    shared |= (s[2] != ld and at < s[1] and s[0] < place[-1] + 1
                               and (written or s[3]))
                if rows > 1:
                    spans.append((at, int(place[-1]) + 1, ld, written))
        if shared:
            refused += 1
            with pytest.raises(lst.LstError):
                lst.lst_clip(lists[0], 0.5, out=lists[1])
            continue
        taken += 1
        before = [_np(t) for t in lists[0]]
        norm = lst.lst_clip(lists[0], 0.5, out=lists[1])
        _check(before, [t if o is None else o for t, o in zip(*lists)], norm, 0.5)
    assert taken > 40 and refused > 40


def test_many_columns_of_one_matrix_are_compared_quickly():
    """The list's last matrices share memory: refused, in a time far below that of all pairs
    (2^31 of them, seconds)."""
    n = 65_536
    table = (lst.lst_gradient * n)()
    for i, g in enumerate(table):  # never read: the call is refused
        g.data, g.rows, g.cols, g.ld = (1 << 30) + 64 * min(i, n - 2), 500, 16, 16 * n
    lib, p = lst.load_library(), 1 << 20
    start = time.process_time()
    assert lib.lst_clip(n, table, 1.0, p, p, None, None) == lst.LST_EINVAL
    assert time.process_time() - start < 1.0


@pytest.mark.gpu
def test_large(gpu_lib):
    """More tiles than a launch has blocks, and a sum that float32 would not hold."""
    t = torch.full((40_000_003,), 2.0 ** -10, device="cuda")
    s = torch.ones((3000, 4001), device="cuda", dtype=torch.bfloat16)
    half = s[:, :2001]
    norm = lst.lst_clip([t, half], 100.0)
    n = np.sqrt(40_000_003 * 2.0 ** -20 + 3000 * 2001)
    assert abs(float(norm) - n) <= 1.01 * U * n
    f = 100.0 / n
    assert (torch.abs(t - f * 2.0 ** -10) <= 2.01 * U * f * 2.0 ** -10).all()
    assert torch.equal(half, torch.full_like(half, f)) and (s[:, 2001:] == 1).all()


@pytest.mark.gpu
def test_no_matrices(gpu_lib):
    """None at all, by the C entry, and none with an element."""
    norm = torch.ones((), device="cuda")
    work = torch.empty(lst.lst_clip_workspace(0), dtype=torch.uint8, device="cuda")
    assert lst.load_library().lst_clip(0, None, 1.0, norm.data_ptr(), work.data_ptr(), None,
                                       torch.cuda.current_stream().cuda_stream) == lst.LST_OK
    assert float(norm) == 0
    assert float(lst.lst_clip([torch.zeros((3, 0), device="cuda")], 0.0)) == 0


@pytest.mark.gpu
def test_extremes_and_what_is_not_finite(gpu_lib):
    for big in (3e38, 2.0 ** -140):
        t = [torch.full((1000,), big, device="cuda")]
        norm = lst.lst_clip(t, big)
        n = np.sqrt(1000.0) * float(np.float32(big))
        f = float(np.float32(big)) / n
        if big > 1:
            assert torch.isinf(norm).all()  # no float, but the factor is what it is
            assert (torch.abs(t[0].double() - f * big) <= 1e-6 * f * big).all()
        else:
            assert abs(float(norm) - n) <= 2.0 ** -149
            assert (torch.abs(t[0].double() - f * big) <= 2.0 ** -149).all()
    for bad in (float("inf"), float("nan")):
        a, b = torch.randn(50, device="cuda"), torch.randn((9, 9), device="cuda")
        a[7] = bad
        was, out = b.clone(), [torch.zeros_like(a), torch.zeros_like(b)]
        clip = lst.GradientClip([a, b])
        norm = clip.clip(0.1)
        assert clip.sync() == lst.LST_ENONFINITE and clip.sync() == lst.LST_OK
        assert not torch.isfinite(norm).any() and torch.equal(b, was)
        lst.lst_clip([a, b], 0.1, out=out)
        assert torch.equal(out[1], b) and torch.equal(torch.nan_to_num(out[0]), torch.nan_to_num(a))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES[:2])
@pytest.mark.parametrize("big,max_norm", [(1e37, 1e-6), (3e38, 1.0), (3e38, 2.0 ** -30),
                                          (1e30, 2.0 ** -100), (1e38, 1e-100)])
def test_factors_below_normal_floats(gpu_lib, dtype, big, max_norm):
    """Gradients so large that max_norm / n is no normal float: each element within its
    roundings all the same, small ones beside the large ones too."""
    g = torch.Generator("cuda").manual_seed(5)
    a = (torch.rand(300, device="cuda", generator=g) * big).to(dtype)
    b = (torch.randn((9, 17), device="cuda", generator=g) * (big * 2.0 ** -70)).to(dtype)
    c = torch.randn((5, 8), device="cuda", generator=g).to(dtype)
    before = [_np(t) for t in (a, b, c)]
    out = [torch.empty_like(t) for t in (a, b, c)]
    n = norms.clip(before, max_norm)[0]
    assert 0 < max_norm / n < 2.0 ** -126
    for norm, got in ((lst.lst_clip([a, b, c], max_norm, out=out), out),
                      (lst.lst_clip([a, b, c], max_norm), [a, b, c])):
        if n > 3.5e38:
            assert torch.isinf(norm).all()
            norm = torch.tensor(n, dtype=torch.float64)
        _check(before, got, norm, max_norm)


@pytest.mark.gpu
def test_a_factor_whose_fraction_rounds_to_one(gpu_lib):
    t = [torch.full((1,), 2.0 ** 100, device="cuda")]
    lst.lst_clip(t, (1 - 2.0 ** -40) * 2.0 ** -100)
    assert float(t[0]) == 2.0 ** -100


@pytest.mark.gpu
@pytest.mark.parametrize("max_norm", [0.0, 1e-30, 1e-6, 2.0 ** -3])
def test_float16_beside_large_gradients(gpu_lib, max_norm):
    a = torch.full((70,), 2e38, device="cuda")
    b = torch.full((5, 33), 60_000.0, device="cuda", dtype=torch.float16)
    before = [_np(t) for t in (a, b)]
    lst.lst_clip([a, b], max_norm)
    _check(before, [a, b], torch.tensor(norms.clip(before, max_norm)[0], dtype=torch.float64),
           max_norm)
    assert (b == 0).all()


@pytest.mark.gpu
def test_repeats_captures_and_streams(gpu_lib):
    tensors = _tensors([(500, 900), (700,), (33, 65)], 5)
    out = [torch.empty_like(t) for t in tensors]
    clip = lst.GradientClip(tensors, out=out)
    first = float(clip.clip(1.0))
    kept = [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = clip.clip(1.0)
    side.synchronize()
    assert float(again) == first and all(torch.equal(a, b) for a, b in zip(kept, out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = clip.clip(1.0)
    for i in range(4):
        for t in tensors:
            t.copy_(torch.randn(t.shape, device="cuda") * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        _check([_np(t) for t in tensors], out, norm, 1.0)
    assert clip.sync() == lst.LST_OK


def _list(*grads):
    a = (lst.lst_gradient * max(1, len(grads)))()
    for g, kw in zip(a, grads):
        base = dict(data=4096, out=None, rows=2, cols=8, ld=8, ldo=8, dtype=0)
        for k, v in {**base, **kw}.items():
            setattr(g, k, v)
    return a


def test_refusals_on_the_host():
    lib, bad = lst.load_library(), lst.LST_EINVAL
    p = 1 << 20  # never read: every call is refused

    def call(*grads, n=None, max_norm=1.0, norm=p, work=p):
        return lib.lst_clip(len(grads) if n is None else n, _list(*grads), max_norm, norm, work,
                            None, None)

    for kw in (dict(dtype=3), dict(rows=-1), dict(cols=-1), dict(data=None), dict(ld=7),
               dict(out=8192, ldo=7), dict(out=4096, ldo=9), dict(rows=1 << 41),
               dict(cols=1 << 41, ld=1 << 41), dict(rows=1 << 21, cols=1 << 20, ld=1 << 20),
               dict(rows=1 << 20, ld=1 << 40)):
        assert call(kw) == bad, kw
    assert call({}, n=-1) == bad and call({}, n=65_537) == bad
    assert lib.lst_clip(1, None, 1.0, p, p, None, None) == bad
    for kw in (dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norm=None), dict(work=None),
               dict(work=p + 8)):
        assert call({}, **kw) == bad, kw
    # memory that two of them share, one of which is written
    for pair in (({}, {}), ({}, dict(data=4096 + 60)), ({}, dict(data=8192, out=4096 + 32)),
                 (dict(out=8192), dict(data=8192, out=16384)), ({"out": 4096 + 32},),
                 (dict(out=8192), dict(data=12288, out=8192 + 4)),
                 (dict(ld=16), dict(data=4096 + 28, ld=16)),        # a column in both
                 (dict(ld=16), dict(data=4096 + 40, ld=16)),        # wrapped into the next row
                 (dict(ld=16), dict(data=4096 + 32, ld=17))):
        assert call(*pair) == bad, pair
    assert lst.lst_clip_workspace(1) == 8 * 2049 and lst.lst_clip_workspace(61) == 8 * 4097
    assert lib.lst_clip_workspace(-1) == -1 and lib.lst_clip_workspace(65_537) == -1
    assert ctypes.sizeof(lst.lst_gradient) == 56


def test_tensors_on_the_host_are_refused():
    with pytest.raises(TypeError):
        lst.lst_clip([torch.zeros(3)], 1.0)
    with pytest.raises(ValueError):
        lst.lst_clip([], 1.0)


@pytest.mark.gpu
def test_refusals_of_tensors(gpu_lib):
    x = torch.zeros((6, 8), device="cuda")
    for bad in (lambda: lst.lst_clip([x, x], 1.0), lambda: lst.lst_clip([x, x[2:]], 1.0),
                lambda: lst.lst_clip([x.double()], 1.0), lambda: lst.lst_clip([x.t()], 1.0),
                lambda: lst.lst_clip([x.view(2, 3, 8)[:, :2]], 1.0),
                lambda: lst.lst_clip([x], 1.0, out=[x.bfloat16()]),
                lambda: lst.lst_clip([x], 1.0, out=[x[:5]]), lambda: lst.lst_clip([x], -1.0),
                lambda: lst.lst_clip([x], 1.0, out=[]), lambda: lst.lst_clip([x, x.cpu()], 1.0),
                lambda: lst.lst_clip([x[:, :5]], 1.0, out=[x[:, 3:]])):
        with pytest.raises((TypeError, ValueError, lst.LstError)):
            bad()
    # both read, neither written
    out = [torch.empty_like(x) for _ in range(2)]
    lst.lst_clip([x + 1, x + 1], 1.0, out=out)
    y = x + 1
    norm = lst.lst_clip([y, y], 1.0, out=out)
    assert abs(float(norm) - np.sqrt(96)) < 1e-5
