"""lst_logprobs and lst_logprobs_backward against oracle.answers: the likeliest tokens exactly,
logarithms, entropies and gradients within their roundings."""
import numpy as np
import pytest
import torch

import paper_1412_7091_amd as lst
from oracle import answers

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24
INF = float("inf")


def _np(t):
    return t.detach().double().cpu().numpy()


def _dev(a, dtype=torch.float32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def _logits(m, D, dtype, spread=3.0, masked=0.05):
    g = torch.Generator("cuda").manual_seed(m * 100_000 + D)
    x = torch.randn((m, D), device="cuda", generator=g) * spread
    x[torch.rand((m, D), device="cuda", generator=g) < masked] = -INF
    return x.to(dtype)


def _sum_bar(D, reach):
    """How far a float32 sum of D weights, and what is behind it, may be off, relative to it: a
    thread's chain of at most 64 entries a pass of the block, the joins (32 more), and each
    weight's own: the difference, its product with log2(e) / T (rounded itself) and the
    instruction's 2 units, where an exponent of `reach` counts each rounding that many times."""
    return U * (32 + 64 + D / 2048 * 0.05 + 4 + 3 * reach)


def _check_row(x, i, tokens, t, got, top):
    D = len(x)
    logp, h, ids, best = answers.logprobs(x, tokens, t, top)
    fine = np.isfinite(x)
    z = (x[fine] - x[fine].max()) / t if fine.any() and 0 < t < np.inf else np.zeros(1)
    w = np.exp(z)
    p = w / w.sum()
    # the exponent's roundings count by what the weights of each exponent sum to
    reach = 1 + (p * np.abs(z)).sum()
    bar = _sum_bar(D, reach)
    have = _np(got[0])[i]
    assert np.array_equal(np.isfinite(have), np.isfinite(logp)), i
    some = np.isfinite(logp)
    # the quotient of a rounded difference, the logarithm (2 units) and the last difference
    off = bar + U * (4 * np.abs(logp[some]) + 8 + 2 * np.log(D + 1))
    assert (np.abs(have[some] - logp[some]) <= off).all(), i
    # log S and the mean of z, which cancel
    mean = (p * np.abs(z)).sum()
    second = (p * z * z).sum()
    off = 2 * bar * (1 + mean) + U * (8 * mean + 4 * second + 2 * np.log(D + 1) + 4)
    assert abs(float(got[1][i]) - h) <= off, i
    if top:
        assert np.array_equal(got[2][i].cpu().numpy(), ids), i
        have = _np(got[3])[i]
        assert np.array_equal(np.isfinite(have), np.isfinite(best))
        some = np.isfinite(best)
        off = bar + U * (4 * np.abs(best[some]) + 8 + 2 * np.log(D + 1))
        assert (np.abs(have[some] - best[some]) <= off).all(), i


def _check_grad(x, i, tokens, t, g, ge, got, dtype):
    D = len(x)
    want = answers.logprobs_grad(x, tokens, g, ge, t)
    fine = np.isfinite(x)
    if not fine.any():
        assert (_np(got)[i] == 0).all()
        return
    z = np.where(fine, (np.where(fine, x, 0) - x[fine].max()) / t, 0)
    w = np.where(fine, np.exp(z), 0)
    p = w / w.sum()
    log = np.where(p > 0, z - np.log(w.sum()), 0)
    reach = 1 + (p * np.abs(z)).sum()
    bar = _sum_bar(D, reach)
    h = -(p * log).sum()
    used = np.array([0 <= k < D and np.isfinite(x[k]) for k in tokens], dtype=bool)
    size = np.abs(g[used]).sum()
    inner = size + abs(ge) * (np.abs(log) + h)
    own = np.zeros(D)
    for k, v in zip(np.asarray(tokens)[used], np.abs(g[used])):
        own[k] += v
    # the weight's exponent counts its roundings |z| times; the entropy's own bar is 2 bar (1 + h)
    off = p * (inner * (bar + U * (12 + 4 * np.abs(z))) + abs(ge) * (3 * bar * (2 + h))
               + size * U * len(tokens)) + own * U * (len(tokens) + 3) + np.abs(want) * t * 3 * U
    off = off / t + torch.finfo(dtype).eps / 2 * np.abs(want) * 1.01 + 2.0 ** -126
    if dtype == torch.float16:
        off += 2.0 ** -25
    assert (np.abs(_np(got)[i] - want) <= off).all(), i


def _tokens(rng, m, K, D):
    tokens = rng.integers(0, D, (m, K))
    tokens[rng.random((m, K)) < 0.1] = -1
    if K > 2:
        tokens[:, 2] = tokens[:, 0]  # the same token twice
    return tokens


def _run(m, D, K, top, dtype, temperature, spread=3.0):
    rng = np.random.default_rng(m * 7 + D + K)
    x = _logits(m, D, dtype, spread)
    tokens = _tokens(rng, m, K, D)
    t = rng.uniform(0.5, 1.5, m).astype(np.float32) if temperature else np.ones(m, np.float32)
    tt = _dev(t) if temperature else None
    td = _dev(tokens, torch.int32)
    got = lst.lst_logprobs(x, td, top=top, temperature=tt, save=True)
    g, ge = rng.standard_normal((m, K)).astype(np.float32), rng.standard_normal(m).astype(np.float32)
    grad = lst.lst_logprobs_backward(x, td, got[4], _dev(g), _dev(ge), temperature=tt)
    plain = lst.lst_logprobs_backward(x, td, got[4], _dev(g), temperature=tt)
    X = _np(x)
    for i in range(m) if m <= 8 else sorted({0, 1, m // 2, m - 1}):
        _check_row(X[i], i, tokens[i], float(t[i]), got, top)
        _check_grad(X[i], i, tokens[i], float(t[i]), g[i], float(ge[i]), grad, dtype)
        _check_grad(X[i], i, tokens[i], float(t[i]), g[i], 0.0, plain, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("m,D,K,top", [
    (1, 1, 1, 1), (3, 7, 2, 5), (2, 8, 1, 8), (4, 127, 3, 3), (5, 128, 1, 1), (2, 129, 1, 64),
    (7, 1000, 10, 20), (3, 4096, 5, 0), (2, 4097, 1, 33), (6, 16384, 4, 7), (2, 16385, 3, 64),
    (1, 16386, 1, 2), (3, 50_000, 16, 20), (40, 20_001, 1, 5), (1, 1_000_003, 2, 32),
    (300, 60_000, 1, 1), (2, 5, 1, 9), (1, 1_100_001, 2, 64), (1, 1_048_576, 1, 20)])
def test_float32(gpu_lib, m, D, K, top):
    _run(m, D, K, top, torch.float32, False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,D,K,top", [(3, 500, 3, 5), (4, 9001, 6, 20), (2, 100_001, 2, 50),
                                       (130, 130_003, 3, 5)])
@pytest.mark.parametrize("spread", [0.0, 0.4, 6.0])
def test_types_temperatures_and_ties(gpu_lib, dtype, m, D, K, top, spread):
    _run(m, D, K, top, dtype, True, spread)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [60, 30_000])
def test_masks_and_what_is_not_finite(gpu_lib, D):
    """Rows without an entry, of the type's lowest value, with infinities and no numbers; very
    large and very small entries; bad temperatures."""
    rng = np.random.default_rng(D)
    low = torch.finfo(torch.float32).min
    x = rng.standard_normal((14, D)).astype(np.float32)
    x[0] = -INF
    x[1] = np.nan
    x[2] = low
    x[3, 1:] = low
    x[4, 5] = INF
    x[5, [3, D - 1]] = INF
    x[6, ::2] = np.nan
    x[7, :D // 2] = -INF
    x[7, 3] = -2.0
    x[8] = -INF
    x[8, D - 2] = 1e30
    x[9] *= 1e30
    x[10] += 3e4
    x[11] = 3e38
    x[12, ::2] = -3e38
    tokens = np.tile(np.array([3, 5, D - 1, D - 2, 0, -1]), (14, 1))
    td = _dev(tokens, torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = lst.lst_logprobs(_dev(x), td, top=10, save=True, status=status)
    g = rng.standard_normal(tokens.shape).astype(np.float32)
    ge = np.ones(14, np.float32)
    grad = lst.lst_logprobs_backward(_dev(x), td, got[4], _dev(g), _dev(ge))
    assert int(status) == 0
    for i in range(14):
        logp, h, ids, best = answers.logprobs(x[i], tokens[i], 1.0, 10)
        have = _np(got[0])[i]
        assert np.array_equal(have == -INF, logp == -INF), i
        some = np.isfinite(logp)
        size = np.abs(logp[some]) * 4 * U + 2e-6  # far above _sum_bar of these sizes
        assert (np.abs(have[some] - logp[some]) <= size).all(), i
        assert abs(float(got[1][i]) - h) <= 4e-6, i
        assert np.array_equal(got[2][i].cpu().numpy(), ids), i
        want = answers.logprobs_grad(x[i].astype(np.float64), tokens[i], g[i], 1.0)
        assert (np.abs(_np(grad)[i] - want) <= 2e-5 * (1 + np.abs(want))).all(), i
        if i not in (4, 5):
            assert (_np(grad)[i][~(x[i] > -INF)] == 0).all(), i
    for t in (0.0, -1.0, INF, np.nan):
        got = lst.lst_logprobs(_dev(x[9:]), td[9:], top=2, save=True,
                               temperature=torch.full((5,), t, device="cuda"))
        assert (got[0][:, :5] == -INF).all() and (got[0][:, 5] == 0).all()
        assert (got[1] == 0).all() and (got[2] == -1).all() and (got[3] == -INF).all()
        grad = lst.lst_logprobs_backward(_dev(x[9:]), td[9:], got[4], _dev(g[9:]),
                                         temperature=torch.full((5,), t, device="cuda"))
        assert (grad == 0).all()
    # temperatures at the ends of what there is: all on the largest, or none left out
    t = torch.tensor([1e-40, 1e-30, 1e30, 3e38], device="cuda")
    y = _dev(rng.standard_normal((4, D)))
    got = lst.lst_logprobs(y, top=1, temperature=t)
    assert torch.equal(got[2][:, 0].long(), y.argmax(dim=1))
    assert (got[1][:2] == 0).all() and (got[3][:2] == 0).all()
    assert (torch.abs(got[1][2:] - np.log(D)) < 1e-4).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES[:2])
@pytest.mark.parametrize("D", [2, 60, 9001, 30_000, 200_003])
def test_entries_further_apart_than_the_largest_float(gpu_lib, dtype, D):
    """Entries near both ends of the type at temperatures that leave them all a probability: the
    sums, the tokens' logarithms and the gradient go by the same exponents."""
    rng = np.random.default_rng(D)
    x = rng.uniform(-3.3e38, 3.3e38, (5, D))
    x[:, 0], x[:, 1] = 3.3e38, -3.3e38
    x[1, D // 2:] = -3.3e38
    x[2, 1:D // 2 + 1], x[2, D // 2 + 1:] = -3.3e38, 3.3e38
    x[3, 2:][rng.random(max(0, D - 2)) < 0.5] = -INF
    x[4, 2:] = -3.2e38
    x = _dev(x, dtype)
    t = np.array([1e38, 1e38, 1e38, 3e37, 1e36], np.float32)
    tokens = np.tile(np.array([1, 0, D - 1, -1]), (5, 1))
    td, tt = _dev(tokens, torch.int32), _dev(t)
    # a gradient of ordinary size: it is divided by the temperature
    g, ge = rng.standard_normal((5, 4)).astype(np.float32) * np.float32(1e33), np.full(
        5, 1e33, np.float32)
    got = lst.lst_logprobs(x, td, top=5, temperature=tt, save=True)
    grad = lst.lst_logprobs_backward(x, td, got[4], _dev(g), _dev(ge), temperature=tt)
    for i, row in enumerate(_np(x)):
        _check_row(row, i, tokens[i], float(t[i]), got, 5)
        _check_grad(row, i, tokens[i], float(t[i]), g[i], float(ge[i]), grad, dtype)


@pytest.mark.gpu
def test_indices_outside_set_the_status(gpu_lib):
    x = _logits(2, 40, torch.float32, masked=0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    td = _dev([[1, 40], [-2, 39]], torch.int32)
    logp, _, _, _, saved = lst.lst_logprobs(x, td, save=True, status=status)
    assert int(status) == lst.LST_EINDEX
    assert logp[0, 1] == 0 and logp[1, 0] == 0 and logp[0, 0] < 0 and logp[1, 1] < 0
    g = torch.full((2, 2), 1.0, device="cuda")
    clean = _dev([[1, -1], [-1, 39]], torch.int32)
    want = lst.lst_logprobs_backward(x, clean, lst.lst_logprobs(x, clean, save=True)[4], g)
    assert torch.equal(lst.lst_logprobs_backward(x, td, saved, g), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [333, 40_000])
def test_strides_in_place_and_what_is_beside(gpu_lib, dtype, D):
    m, K = 5, 6
    rng = np.random.default_rng(1)
    x = _logits(m, D, dtype)
    whole = torch.randn((m, 2 * D + 5), device="cuda").to(dtype)
    view = whole[:, 3:3 + D]
    view.copy_(x)
    was = whole.clone()
    tokens = _dev(_tokens(rng, m, K, D), torch.int32)
    want = lst.lst_logprobs(x, tokens, top=9, save=True)
    got = lst.lst_logprobs(view, tokens, top=9, save=True)
    assert all(torch.equal(a, b) or torch.equal(a.isnan(), b.isnan()) for a, b in zip(want, got))
    g = _dev(rng.standard_normal((m, K)))
    grad = lst.lst_logprobs_backward(x, tokens, want[4], g)
    assert torch.equal(grad, lst.lst_logprobs_backward(view, tokens, got[4], g, out=view))
    assert torch.equal(view, grad)
    whole[:, 3:3 + D], was[:, 3:3 + D] = 0, 0
    assert torch.equal(whole, was)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [1500, 70_000])
def test_many_tokens_of_one_place(gpu_lib, D):
    """1024 tokens a row, most of them the same few."""
    rng = np.random.default_rng(6)
    x = _logits(3, D, torch.float32, masked=0)
    tokens = rng.integers(D - 5, D, (3, 1024))
    g = rng.standard_normal((3, 1024)).astype(np.float32)
    td = _dev(tokens, torch.int32)
    got = lst.lst_logprobs(x, td, save=True)
    grad = lst.lst_logprobs_backward(x, td, got[4], _dev(g))
    for i in range(3):
        _check_row(_np(x)[i], i, tokens[i], 1.0, got, 0)
        _check_grad(_np(x)[i], i, tokens[i], 1.0, g[i], 0.0, grad, torch.float32)
    again = lst.lst_logprobs_backward(x, td, got[4], _dev(g))
    assert torch.equal(grad, again)


@pytest.mark.gpu
def test_more_rows_than_a_batch_of_launches(gpu_lib):
    """66 000 rows of 16 400: the second batch of both directions, and the rows around its begin."""
    m, D = 66_000, 16_400
    batch = 0xFFFFFF // 9
    assert batch > m and (1 << 30) // D < m  # the second is what bounds a batch
    first = (1 << 30) // D
    x = torch.zeros((m, D), device="cuda", dtype=torch.bfloat16)
    rows = [0, first - 1, first, first + 1, m - 1]
    part = torch.randn((5, D), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    x[rows] = part.bfloat16()
    td = torch.full((m, 1), 7, dtype=torch.int32, device="cuda")
    got = lst.lst_logprobs(x, td, top=2, save=True)
    g, ge = torch.ones((m, 1), device="cuda"), torch.full((m,), 0.5, device="cuda")
    want = lst.lst_logprobs(x[rows].contiguous(), td[:5].contiguous(), top=2, save=True)
    for a, b in zip(got, want):
        assert torch.equal(a[rows], b)
    flat = torch.ones(m, dtype=torch.bool, device="cuda")
    flat[rows] = False
    assert (torch.abs(got[0][flat] + np.log(D)) < 1e-5).all()
    assert (got[2][flat] == torch.tensor([0, 1], device="cuda", dtype=torch.int32)).all()
    small = lst.lst_logprobs_backward(x[rows].contiguous(), td[:5].contiguous(), want[4], g[:5],
                                      ge[:5])
    grad = lst.lst_logprobs_backward(x, td, got[4], g, ge, out=x)
    assert torch.equal(grad[rows], small)


@pytest.mark.gpu
def test_shapes_without_tokens_or_rows(gpu_lib):
    x = _logits(4, 90, torch.bfloat16)
    logp, h, ids, best, saved = lst.lst_logprobs(x)
    assert logp is None and ids is None and best is None and saved is None and h.shape == (4,)
    one = lst.lst_logprobs(x, _dev([1, 2, 3, 4], torch.int32))[0]
    assert one.shape == (4,)
    none = lst.lst_logprobs(x[:0], _dev(np.zeros((0, 2)), torch.int32), top=3, save=True)
    assert none[0].shape == (0, 2) and none[2].shape == (0, 3)
    # the entropy's gradient alone
    _, _, _, _, saved = lst.lst_logprobs(x, save=True)
    grad = lst.lst_logprobs_backward(x, None, saved, None, torch.ones(4, device="cuda"))
    for i in range(4):
        _check_grad(_np(x)[i], i, np.zeros(0, int), 1.0, np.zeros(0), 1.0, grad, torch.bfloat16)


@pytest.mark.gpu
def test_gradient_against_differences(gpu_lib):
    rng = np.random.default_rng(9)
    x = _logits(1, 300, torch.float32)
    tokens, t = np.array([[5, 17, 5, -1]]), torch.full((1,), 0.7, device="cuda")
    g, ge = rng.standard_normal((1, 4)), np.array([0.5])
    td = _dev(tokens, torch.int32)
    saved = lst.lst_logprobs(x, td, temperature=t, save=True)[4]
    grad = _np(lst.lst_logprobs_backward(x, td, saved, _dev(g), _dev(ge), temperature=t))[0]
    X = _np(x)[0]
    alive = np.isfinite(X)

    def total(y):
        logp, h, _, _ = answers.logprobs(y, tokens[0], float(t[0]))
        return (np.where(np.isfinite(logp), logp, 0) * g[0]).sum() + 0.5 * h

    for _ in range(4):
        u = np.where(alive, rng.standard_normal(300), 0.0)
        slope = (total(X + 1e-6 * u) - total(X - 1e-6 * u)) / 2e-6
        assert abs(slope - (grad * u).sum()) < 1e-5 * np.linalg.norm(grad) * np.linalg.norm(u)


@pytest.mark.gpu
def test_of_a_layer_and_with_the_chosen_token(gpu_lib):
    """The log probability of what lst_sample chose, without a filter, is that of its prob."""
    g = torch.Generator("cuda").manual_seed(5)
    W = torch.randn((5000, 64), device="cuda", generator=g)
    H = torch.randn((9, 64), device="cuda", generator=g)
    for held in (lst.EightBitOutputLayer(W), lst.FourBitOutputLayer(W)):
        t = torch.full((9,), 5.0, device="cuda")
        u = torch.rand(9, device="cuda", generator=g)
        tokens, prob = held.sample(H, u, temperature=t)
        logp, _, ids, best, _ = held.logprobs(H, tokens, top=1, temperature=t)
        assert (torch.abs(logp - torch.log(prob)) < 1e-5).all()
        assert torch.equal(ids[:, 0].long(), held.scores(H).argmax(dim=1))


@pytest.mark.gpu
@pytest.mark.parametrize("D", [900, 50_000])
def test_captured_and_on_another_stream(gpu_lib, D):
    m, K = 6, 3
    x = _logits(m, D, torch.float32)
    rng = np.random.default_rng(4)
    td, g = _dev(_tokens(rng, m, K, D), torch.int32), _dev(rng.standard_normal((m, K)))
    both = lambda: lst.lst_logprobs(x, td, top=5, save=True)  # noqa: E731
    lst.lst_logprobs_backward(x, td, both()[4], g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
        grad = lst.lst_logprobs_backward(x, td, got[4], g)
    for i in range(4):
        x.copy_(torch.randn_like(x) * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        have = [t.clone() for t in (*got, grad)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            e = both()
            want = (*e, lst.lst_logprobs_backward(x, td, e[4], g))
        side.synchronize()
        for a, b in zip(have, want):
            assert torch.equal(torch.nan_to_num(a.float(), 7.0), torch.nan_to_num(b.float(), 7.0))


def test_refusals_on_the_host():
    lib, ok, bad = lst.load_library(), lst.LST_OK, lst.LST_EINVAL
    p = 4096  # never read: every call is refused, or has no rows

    def forward(dtype=0, m=2, D=9, K=1, top=0, x=p, ldx=9, tokens=p, logp=p, ids=None, best=None,
                work=None):
        return lib.lst_logprobs(dtype, m, D, K, top, x, ldx, None, tokens, logp, None, ids, best,
                                None, work, None, None)

    assert forward(m=0) == ok
    for kw in (dict(dtype=3), dict(m=-1), dict(D=0), dict(D=(1 << 30) + 1, ldx=1 << 31),
               dict(K=-1), dict(K=1025), dict(top=-1), dict(top=65, ids=p, best=p), dict(x=None),
               dict(ldx=8), dict(tokens=None), dict(logp=None), dict(top=1, ids=p),
               dict(top=1, best=p), dict(D=20_000, ldx=20_000),
               dict(D=20_000, ldx=20_000, work=p + 8)):
        assert forward(**kw) == bad, kw

    def backward(dtype=0, m=2, D=9, K=1, x=p, ldx=9, tokens=p, saved=p, g=p, out=p, ldg=9):
        return lib.lst_logprobs_backward(dtype, m, D, K, x, ldx, None, tokens, saved, g, None, out,
                                         ldg, None)

    assert backward(m=0) == ok
    for kw in (dict(dtype=3), dict(m=-1), dict(D=0), dict(K=1025), dict(x=None), dict(ldx=8),
               dict(tokens=None), dict(saved=None), dict(g=None), dict(out=None), dict(ldg=8),
               dict(ldg=10)):
        assert backward(**kw) == bad, kw
    assert lib.lst_logprobs_workspace(1, 0, 0) == -1 and lib.lst_logprobs_workspace(1, 5, 65) == -1
    assert lib.lst_logprobs_workspace(3, 16_384, 5) == 0
    assert lib.lst_logprobs_workspace(3, 20_000, 0) == 3 * 10 * 16
    assert lib.lst_logprobs_saved(3, 5) == 27 and lib.lst_logprobs_saved(3, 1025) == -1


@pytest.mark.gpu
def test_refusals_of_tensors(gpu_lib):
    x = torch.zeros((4, 6), device="cuda")
    t = torch.zeros((4, 1), dtype=torch.int32, device="cuda")
    saved = lst.lst_logprobs(x, t, save=True)[4]
    g = torch.zeros((4, 1), device="cuda")
    for bad in (lambda: lst.lst_logprobs(x.cpu(), t), lambda: lst.lst_logprobs(x.double(), t),
                lambda: lst.lst_logprobs(x, t.long()), lambda: lst.lst_logprobs(x, t[:3]),
                lambda: lst.lst_logprobs(x, t, temperature=g[:2, 0]),
                lambda: lst.lst_logprobs(x, t, top=65), lambda: lst.lst_logprobs(x, t, top=-1),
                lambda: lst.lst_logprobs(x.t(), t),
                lambda: lst.lst_logprobs_backward(x, t, None, g),
                lambda: lst.lst_logprobs_backward(x, t, saved[:2], g),
                lambda: lst.lst_logprobs_backward(x, t, saved, g.bfloat16()),
                lambda: lst.lst_logprobs_backward(x, t, saved, None),
                lambda: lst.lst_logprobs_backward(x, t, saved, g, out=x.bfloat16())):
        with pytest.raises((TypeError, ValueError, lst.LstError)):
            bad()
