"""lst_recur_* against oracle.between, which also bounds what float32 may be off."""
import numpy as np
import pytest
import torch

import paper_1412_7091_amd as lst
from oracle import between

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _np(t):
    return t.detach().double().cpu().numpy()


def _check(got, want, err, dtype=torch.float32):
    off = np.abs(_np(got) - want)
    # 2^-120: exp(-|g|) below the smallest normal float counts as zero, times at most 64
    bar = err + torch.finfo(dtype).eps / 2 * (np.abs(want) + err) + 2.0 ** -120
    if dtype == torch.float16:
        bar = bar + 2.0 ** -25  # half a step of its smallest numbers
    assert (off <= bar).all(), (np.nanmax(off / np.maximum(bar, 1e-300)), off.max())


def _inputs(lengths, d, dtype, seed, gates=1.0, lead=0, behind=0):
    """x and g as the halves of one matrix, offsets, and the rest; rows in no sequence are NaN."""
    g = torch.Generator("cuda").manual_seed(seed)
    off = np.concatenate([[0], np.cumsum(lengths)]) + lead
    n = int(off[-1]) + behind
    z = torch.randn((n, 2 * d), device="cuda", generator=g)
    z[:, d:] = z[:, d:] * gates + gates
    z[:lead], z[int(off[-1]):] = float("nan"), float("nan")
    z = z.to(dtype)
    dy = torch.randn((n, d), device="cuda", generator=g).to(dtype)
    h0, dlast = (torch.randn((len(lengths), d), device="cuda", generator=g) for _ in range(2))
    return z[:, :d], z[:, d:], off, dy, h0, dlast


def _check_all(x, g, off, dy, h0, dlast, offsets="device"):
    dtype, (n, d) = x.dtype, x.shape
    layer = lst.GatedRecurrence(d)
    at = None if offsets is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    n_seq = len(off) - 1
    mark = torch.full((n, d), 7.0, device="cuda").to(dtype)
    y, last, saved = layer.forward(x, g, at, h0, n_seq=n_seq, out=mark.clone(), save=True)
    dx, dg, dh0 = layer.backward(x, g, dy, saved, at, h0, dlast, n_seq=n_seq,
                                 out=(mark.clone(), mark.clone()))
    assert layer.sync() == 0
    own = slice(off[0], off[-1])
    for t in (y, dx, dg):  # rows in no sequence are left as they were
        rest = torch.cat((t[:off[0]], t[off[-1]:]))
        assert (rest == 7).all()
    h0_, dl_ = (None if t is None else _np(t) for t in (h0, dlast))
    wy, wl, ey, el, _ = between.recur(_np(x), _np(g), off, h0_)
    _check(y[own], wy[own], ey[own], dtype)
    _check(last, wl, el)
    (wx, wg, w0), (ex, eg, e0) = between.recur_grad(_np(x), _np(g), off, _np(dy), h0_, dl_)
    _check(dx[own], wx[own], ex[own], dtype)
    _check(dg[own], wg[own], eg[own], dtype)
    _check(dh0, w0, e0)
    return y, last, dx, dg, dh0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,d", [
    ((1,), 1), ((2, 1), 3), ((5, 0, 0, 3, 1), 64), ((0, 0, 4), 65), ((7, 0), 66),
    ((127, 1, 128, 129), 20), ((16, 16, 15, 17, 1, 31), 130), ((300,), 37),
    (tuple([1] * 200), 33), ((0, 140, 0, 0, 260, 2), 500)])
def test_sequences(gpu_lib, dtype, lengths, d):
    _check_all(*_inputs(lengths, d, dtype, 1000 + d))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths", [(6500,), (2047, 2, 2050, 1), (100, 4999)])
def test_long(gpu_lib, dtype, lengths):
    """Sequences over many chunks; gates that keep a state over hundreds of rows."""
    _check_all(*_inputs(lengths, 70, dtype, 77, gates=3.0))


@pytest.mark.gpu
@pytest.mark.parametrize("lead,behind", [(0, 5), (3, 0), (130, 131)])
def test_rows_in_no_sequence(gpu_lib, lead, behind):
    _check_all(*_inputs((4, 0, 150, 9), 36, torch.bfloat16, 5, lead=lead, behind=behind))


@pytest.mark.gpu
def test_without_offsets_and_states(gpu_lib):
    x, g, off, dy, _, _ = _inputs((50, 50, 50), 24, torch.float32, 9)
    _check_all(x, g, off, dy, None, None, offsets=None)
    _check_all(x, g, off, dy, None, None)


@pytest.mark.gpu
def test_no_rows(gpu_lib):
    layer = lst.GatedRecurrence(8)
    x = torch.empty((0, 8), device="cuda")
    h0, off = torch.randn((3, 8), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    y, last, saved = layer.forward(x, x, off, h0, save=True)
    assert torch.equal(last, h0)
    dlast = torch.randn_like(h0)
    dx, dg, dh0 = layer.backward(x, x, x, saved, off, h0, dlast)
    assert torch.equal(dh0, dlast) and layer.sync() == 0
    y, last, _ = layer.forward(x, x, off[:1])
    assert last.shape == (0, 8)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_unaligned_rows(gpu_lib, dtype):
    """Rows at odd strides and addresses, in and out."""
    d, lengths = 50, (9, 140)
    x0, g0, off, dy0, h0, dlast = _inputs(lengths, d, dtype, 31)
    at = torch.tensor(off, dtype=torch.int32, device="cuda")
    want = lst.lst_recur_forward(x0, g0, at, h0, save=True)
    wgrad = lst.lst_recur_backward(x0, g0, dy0, want[2], at, h0, dlast)

    def odd(t):
        big = torch.zeros((t.shape[0], d + 7), device="cuda", dtype=dtype)
        big[:, 3:3 + d] = t
        return big[:, 3:3 + d]

    x, g, dy = odd(x0), odd(g0), odd(dy0)
    y, last, saved = lst.lst_recur_forward(x, g, at, h0, out=odd(x0), save=True)
    dx, dg, dh0 = lst.lst_recur_backward(x, g, dy, saved, at, h0, dlast, out=(odd(x0), odd(x0)))
    for a, b in zip((y, last, dx, dg, dh0), (want[0], want[1], *wgrad)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_saturated_gates(gpu_lib):
    """Gates far out: nothing comes in or nothing stays; infinite gates do so exactly."""
    n, d = 40, 12
    x = torch.randn((n, d), device="cuda")
    g = torch.zeros((n, d), device="cuda")
    g[:, 0], g[:, 1], g[:, 2], g[:, 3] = 90.0, -90.0, float("inf"), -float("inf")
    g[:, 4], g[:, 5], g[:, 6], g[:, 7] = 17.0, -17.0, 200.0, -200.0
    h0 = torch.randn((1, d), device="cuda")
    off = np.array([0, n])
    y, last, dx, dg, dh0 = _check_all(x, g, off, torch.randn_like(x), h0, torch.randn_like(h0))
    assert torch.equal(y[:, 2], h0[0, 2].expand(n)) and torch.equal(y[:, 3], x[:, 3])
    assert (dg[:, 2:4] == 0).all()


@pytest.mark.gpu
def test_not_a_number_stays_in_its_sequence(gpu_lib):
    x, g, off, dy, h0, dlast = _inputs((30, 200, 40), 40, torch.float32, 6)
    at = torch.tensor(off, dtype=torch.int32, device="cuda")
    y0 = lst.lst_recur_forward(x, g, at, h0)[0]
    g[100, 5] = float("nan")
    # a quiet number with every bit set, and one with a payload
    g.view(torch.int32)[120, 6] = -1
    x.view(torch.int32)[35, 7] = 0x7FC12345
    y, last, _ = lst.lst_recur_forward(x, g, at, h0)
    for ch, row in ((5, 100), (6, 120), (7, 35)):
        assert y[row:230, ch].isnan().all() and not y[:row, ch].isnan().any()
        assert last[1, ch].isnan()
    ok = torch.ones(40, dtype=torch.bool)
    ok[5:8] = False
    assert torch.equal(y[:, ok], y0[:, ok]) and torch.equal(y[230:], y0[230:])


@pytest.mark.gpu
def test_last_state_in_place_and_continued(gpu_lib):
    """A sequence in two calls, the state handed on in one buffer, is the sequence in one."""
    x, g, off, _, h0, _ = _inputs((600,), 48, torch.float32, 8)
    whole, last, _ = lst.lst_recur_forward(x, g, None, h0)
    h = h0.clone()
    first, _, _ = lst.lst_recur_forward(x[:100], g[:100], None, h, h_last=h)
    rest, _, _ = lst.lst_recur_forward(x[100:], g[100:], None, h, h_last=h)
    _, wl, ey, el, _ = between.recur(_np(x), _np(g), off, _np(h0))
    assert np.abs(_np(torch.cat((first, rest)) - whole)).max() <= 2 * ey.max()
    assert np.abs(_np(h) - wl).max() <= el.max() + 2.0 ** -24 * np.abs(wl).max()


@pytest.mark.gpu
def test_bad_offsets_set_the_status(gpu_lib):
    x, g, _, dy, _, _ = _inputs((300,), 16, torch.float32, 4)
    layer = lst.GatedRecurrence(16)
    for off in ([0, 200, 100, 300], [-1, 5, 9, 300], [0, 5, 6, 301], [400, 500, 600, 700],
                [300, 200, 100, 0]):
        at = torch.tensor(off, dtype=torch.int32, device="cuda")
        y, _, saved = layer.forward(x, g, at, save=True)
        assert layer.sync() == lst.LST_EINDEX, off
        layer.backward(x, g, dy, saved, at)
        assert layer.sync() == lst.LST_EINDEX and layer.sync() == 0, off


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 65), (64, 500), (700, 33), (2, 4096)])
def test_step(gpu_lib, dtype, rows, d):
    slots = rows + 5
    g = torch.Generator("cuda").manual_seed(rows + d)
    z = torch.randn((rows, 2 * d), device="cuda", generator=g).to(dtype)
    x, gate = z[:, :d], z[:, d:]
    h = torch.randn((slots, d), device="cuda", generator=g)
    at = torch.randperm(slots, device="cuda", generator=g)[:rows].int()
    before = h.clone()
    layer = lst.GatedRecurrence(d)
    y = layer.step(x, gate, h, at)
    assert layer.sync() == 0
    off = np.arange(rows + 1)
    wy, wl, ey, el, _ = between.recur(_np(x), _np(gate), off, _np(before[at.long()]))
    _check(y, wy, ey, dtype)
    _check(h[at.long()], wl, el)
    rest = torch.ones(slots, dtype=torch.bool, device="cuda")
    rest[at.long()] = False
    assert torch.equal(h[rest], before[rest])
    # without slots: row i continues state i; the same numbers
    h2 = before[at.long()].contiguous()
    assert torch.equal(layer.step(x, gate, h2), y) and torch.equal(h2, h[at.long()])


@pytest.mark.gpu
def test_step_is_one_row_of_a_sequence(gpu_lib):
    x, g, off, _, h0, _ = _inputs((5,), 90, torch.float32, 14)
    whole = lst.lst_recur_forward(x, g, None, h0)[0]
    h = h0.clone()
    for t in range(5):
        y = lst.lst_recur_step(x[t:t + 1], g[t:t + 1], h)
        assert torch.allclose(y, whole[t:t + 1], rtol=0, atol=2.0 ** -20)


@pytest.mark.gpu
def test_step_slots_refused(gpu_lib):
    """-1 is no state; indices outside and repeated ones set the status and do nothing."""
    d = 40
    layer = lst.GatedRecurrence(d)
    x, g = (torch.randn((6, d), device="cuda") for _ in range(2))
    h0 = torch.randn((4, d), device="cuda")
    for slots, used, code in (([2, -1, 0, -1, -1, 1], [0, 2, 5], 0),
                              ([2, 4, 0, -2, 1, -1], [0, 2, 4], lst.LST_EINDEX),
                              ([3, 1, 3, 1, 3, 0], [0, 1, 5], lst.LST_EINDEX)):
        h, y = h0.clone(), torch.full((6, d), 7.0, device="cuda")
        layer.step(x, g, h, torch.tensor(slots, dtype=torch.int32, device="cuda"), out=y)
        assert layer.sync() == code
        want = h0.clone()
        for i in used:
            one = h0[slots[i]:slots[i] + 1].clone()
            assert torch.equal(layer.step(x[i:i + 1], g[i:i + 1], one), y[i:i + 1])
            want[slots[i]] = one[0]
        assert torch.equal(h, want)
        idle = [i for i in range(6) if i not in used]
        assert (y[idle] == 7).all()


@pytest.mark.gpu
def test_captured_and_on_two_streams(gpu_lib):
    """Two graphs with passes of their own, replayed in turn and at once."""
    sets = [_inputs((900, 3, 2000), 96, torch.bfloat16, s) for s in (1, 2)]
    graphs, outs, eager = [], [], []

    def both(x, g, off, dy, h0, dlast):
        at = offsets[id(x)]
        y, last, saved = lst.lst_recur_forward(x, g, at, h0, save=True)
        return (y, last, *lst.lst_recur_backward(x, g, dy, saved, at, h0, dlast))

    offsets = {id(s[0]): torch.tensor(s[2], dtype=torch.int32, device="cuda") for s in sets}
    for s in sets:
        eager.append([t.clone() for t in both(*s)])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs.append(both(*s))
        graphs.append(graph)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for st, gr in zip(streams, graphs):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for o, e in zip(outs, eager):
            assert all(torch.equal(a, b) for a, b in zip(o, e))


@pytest.mark.gpu
def test_the_same_call_gives_the_same_bits(gpu_lib):
    x, g, off, dy, h0, dlast = _inputs((3000, 1, 700), 128, torch.float32, 3, gates=2.0)
    at = torch.tensor(off, dtype=torch.int32, device="cuda")
    first = None
    for _ in range(5):
        y, last, saved = lst.lst_recur_forward(x, g, at, h0, save=True)
        got = (y, last, *lst.lst_recur_backward(x, g, dy, saved, at, h0, dlast))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.gpu
def test_refusals(gpu_lib):
    x = torch.zeros((6, 8), device="cuda")
    off = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    layer = lst.GatedRecurrence(8)
    with pytest.raises(ValueError):
        layer.forward(torch.zeros((6, 9), device="cuda"), x, off)
    with pytest.raises(ValueError):
        layer.forward(x, x[:5], off)
    with pytest.raises(TypeError):
        layer.forward(x, x.half(), off)
    with pytest.raises(TypeError):
        layer.forward(x, x, off.long())
    with pytest.raises(TypeError):
        layer.forward(x, x, off.cpu())
    with pytest.raises(ValueError):
        layer.forward(x, x, n_seq=4)
    with pytest.raises(ValueError):
        layer.forward(x, x, off, torch.zeros((2, 8), device="cuda"))
    with pytest.raises(TypeError):
        layer.forward(x.double(), x.double(), off)
    with pytest.raises(ValueError):
        layer.forward(x.T, x.T, off)
    with pytest.raises(ValueError):
        layer.backward(x, x, x, torch.zeros((2, 8), device="cuda"), off)
    with pytest.raises(ValueError):
        layer.step(x, x, torch.zeros((6, 7), device="cuda"))
    with pytest.raises(lst.LstError):
        layer.step(x, x, torch.zeros((5, 8), device="cuda"))
    wide = torch.zeros((2, 4097), device="cuda")
    with pytest.raises(lst.LstError):
        lst.lst_recur_forward(wide, wide)


def test_refusals_on_host():
    lib = lst.load_library()
    P = 16  # never dereferenced

    def forward(dtype=0, rows=4, n=2, d=8, x=P, ldx=8, g=P, ldg=8, off=P, y=P, ldy=8, work=P):
        return lib.lst_recur_forward(dtype, rows, n, d, x, ldx, g, ldg, off, None, y, ldy, None,
                                     None, work, None, None)

    def backward(dtype=0, rows=4, n=2, d=8, x=P, ldx=8, g=P, ldg=8, off=P, y=P, ldy=8, work=P,
                 saved=P, dx=P, ldgx=8, dg=P, ldgg=8):
        return lib.lst_recur_backward(dtype, rows, n, d, x, ldx, g, ldg, off, None, y, ldy, None,
                                      saved, dx, ldgx, dg, ldgg, None, work, None, None)

    bad = [dict(dtype=-1), dict(rows=-1), dict(n=-1), dict(d=0), dict(d=4097), dict(x=None),
           dict(g=None), dict(y=None), dict(ldx=7), dict(ldg=7), dict(ldy=7),
           dict(off=None, n=3), dict(off=None, n=0)]
    for kw in bad:
        assert forward(**kw) == lst.LST_EINVAL, kw
        assert backward(**kw) == lst.LST_EINVAL, kw
    for kw in (dict(saved=None), dict(dx=None), dict(dg=None), dict(ldgx=7), dict(ldgg=7)):
        assert backward(**kw) == lst.LST_EINVAL, kw

    def step(dtype=0, rows=4, n=4, d=8, x=P, ldx=8, g=P, ldg=8, slots=P, h=P, y=P, ldy=8):
        return lib.lst_recur_step(dtype, rows, n, d, x, ldx, g, ldg, slots, h, y, ldy, None, None)

    for kw in (dict(dtype=9), dict(rows=-1), dict(n=-1), dict(d=0), dict(x=None), dict(g=None),
               dict(h=None), dict(y=None), dict(ldx=7), dict(ldg=7), dict(ldy=7),
               dict(slots=None, n=3)):
        assert step(**kw) == lst.LST_EINVAL, kw
    assert step(rows=0) == lst.LST_OK
    assert lst.lst_recur_saved(129, 5) == 10 and lst.lst_recur_saved(-1, 5) == -1
    assert lst.lst_recur_workspace(-1, 5) == -1


def test_sizes_behind_the_limits():
    """Refused on the host: more than 2^30 rows or sequences, whose counts with a block's step
    leave 32 bits, and more slots than each can be compared with."""
    lib = lst.load_library()
    P = 16  # never dereferenced
    for rows, n in (((1 << 30) + 1, 1), (0x7FFFFFFF, 1), (4, (1 << 30) + 1), (4, 0x7FFFFFFF)):
        assert lib.lst_recur_forward(1, rows, n, 1, P, 1, P, 1, P, None, P, 1, None, None, P,
                                     None, None) == lst.LST_EINVAL
        assert lib.lst_recur_backward(1, rows, n, 1, P, 1, P, 1, P, None, P, 1, None, P, P, 1, P,
                                      1, None, P, None, None) == lst.LST_EINVAL
    assert lst.lst_recur_saved((1 << 30) + 1, 1) == lst.lst_recur_saved(1, 4097) == -1
    assert lst.lst_recur_workspace((1 << 30) + 1, 1) == lst.lst_recur_workspace(1, 4097) == -1
    assert lst.lst_recur_saved(1 << 30, 1) == 1 << 23
    for rows, slots in (((1 << 16) + 1, P), (1 << 24, None)):
        assert lib.lst_recur_step(0, rows, 1 << 25, 8, P, 8, P, 8, slots, P, P, 8, None,
                                  None) == lst.LST_EINVAL


@pytest.mark.gpu
def test_widths_refused_with_save(gpu_lib):
    for d in (0, 4097):
        x = torch.zeros(4, d, device="cuda")
        with pytest.raises(lst.LstError):
            lst.lst_recur_forward(x, x, save=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_in_place(gpu_lib, dtype):
    """grad_x and grad_g over the rows of x and g, y over those of x."""
    torch.manual_seed(8)
    rows, d = 700, 66
    x, g, dy = (torch.randn(rows, d, device="cuda").to(dtype) for _ in range(3))
    off = torch.tensor([0, 5, 300, 301, 700], dtype=torch.int32, device="cuda")
    y, _, saved = lst.lst_recur_forward(x, g, off, save=True)
    dx, dg, _ = lst.lst_recur_backward(x, g, dy, saved, off)
    a, b = x.clone(), g.clone()
    lst.lst_recur_backward(a, b, dy, saved, off, out=(a, b))
    assert torch.equal(a, dx) and torch.equal(b, dg)
    a = x.clone()
    lst.lst_recur_forward(a, g, off, out=a)
    assert torch.equal(a, y)


@pytest.mark.gpu
def test_the_most_rows(gpu_lib):
    """2^30 rows, which no single launch has threads for; the rows repeat, and so do the results.
    Sequences of two chunks: one of them lies across the launches' border in each pass."""
    rows, part, d, length = 1 << 30, 1 << 20, 2, 256
    g = torch.Generator("cuda").manual_seed(19)
    x, gate, dy = (torch.randn((part, d), device="cuda", generator=g).bfloat16() for _ in range(3))
    h0, dlast = (torch.randn((part // length, d), device="cuda", generator=g) for _ in range(2))
    many = rows // part
    n = part // length
    y, last, saved = lst.lst_recur_forward(x, gate, None, h0, n_seq=n, save=True)
    want = (y, last, *lst.lst_recur_backward(x, gate, dy, saved, None, h0, dlast, n_seq=n))
    off = np.arange(3) * length
    wy, wl, ey, el, _ = between.recur(_np(x[:512]), _np(gate[:512]), off, _np(h0[:2]))
    _check(y[:512], wy, ey, torch.bfloat16)
    _check(last[:2], wl, el)
    x, gate, dy, h0, dlast = (t.repeat(many, 1) for t in (x, gate, dy, h0, dlast))
    layer = lst.GatedRecurrence(d)
    y, last, saved = layer.forward(x, gate, None, h0, n_seq=many * n, save=True)
    got = (y, last, *layer.backward(x, gate, dy, saved, None, h0, dlast, n_seq=many * n))
    assert layer.sync() == 0
    for a, b in zip(got, want):
        assert bool((a.view(many, *b.shape) == b).all())


def _check_many(lengths, d, dtype, seed):
    """As _check_all, where nearly all of very many sequences have no rows."""
    lengths = np.asarray(lengths)
    x, g, off, dy, h0, dlast = _inputs(lengths, d, dtype, seed)
    layer = lst.GatedRecurrence(d)
    at = torch.tensor(off, dtype=torch.int32, device="cuda")
    y, last, saved = layer.forward(x, g, at, h0, save=True)
    dx, dg, dh0 = layer.backward(x, g, dy, saved, at, h0, dlast)
    assert layer.sync() == 0
    some = lengths > 0
    own = torch.tensor(some, device="cuda")
    assert torch.equal(last[~own], h0[~own]) and torch.equal(dh0[~own], dlast[~own])
    off = np.concatenate([[0], np.cumsum(lengths[some])])
    h0_, dl_ = _np(h0[own]), _np(dlast[own])
    wy, wl, ey, el, _ = between.recur(_np(x), _np(g), off, h0_)
    _check(y, wy, ey, dtype)
    _check(last[own], wl, el)
    (wx, wg, w0), (ex, eg, e0) = between.recur_grad(_np(x), _np(g), off, _np(dy), h0_, dl_)
    _check(dx, wx, ex, dtype)
    _check(dg, wg, eg, dtype)
    _check(dh0[own], w0, e0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(torch.float32, 3), (torch.bfloat16, 6),
                                     (torch.float16, 5)])
@pytest.mark.parametrize("n", [513, 1025, 3000])
def test_more_sequences_than_a_block_has_threads(gpu_lib, dtype, d, n):
    """Sequences of one row; short ones with empty ones among them; runs of empty ones longer
    than a block at the chunks' borders; one sequence of several chunks among short ones."""
    rng = np.random.default_rng(n)
    _check_many(np.ones(n, dtype=int), d, dtype, 1)
    _check_many(rng.integers(0, 4, n), d, dtype, 2)
    gaps = np.zeros(4 * n, dtype=int)
    gaps[[0, n, 2 * n, 3 * n, 4 * n - 1]] = 128, 100, 28, 129, 1
    _check_many(gaps, d, dtype, 3)
    one = rng.integers(0, 2, n)
    one[n // 2] = 700
    _check_many(one, d, dtype, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n", [(torch.float32, 263_000), (torch.bfloat16, 1_060_000)])
def test_sequences_whose_search_takes_two_rounds(gpu_lib, dtype, n):
    rng = np.random.default_rng(n)
    lengths = np.zeros(n, dtype=int)
    lengths[rng.choice(n, 400, replace=False)] = rng.integers(1, 9, 400)
    lengths[[0, n // 3, n - 1]] = 3, 300, 140
    _check_many(lengths, 2, dtype, 5)
    ends = np.zeros(n, dtype=int)
    ends[[0, n - 1]] = 130, 256
    _check_many(ends, 2, dtype, 6)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [600, 1100, 5000])
def test_bad_offsets_among_many_set_the_status(gpu_lib, n):
    x, g, _, dy, _, _ = _inputs((1000,), 16, torch.bfloat16, 4)
    layer = lst.GatedRecurrence(16)
    fine = np.minimum(np.arange(n + 1), 1000)
    fine[-1] = 1000
    down, low, high = fine.copy(), fine.copy(), fine.copy()
    down[n // 2], low[1], high[n // 3:] = 0, -7, 2000
    for off, code in ((fine, 0), (down, lst.LST_EINDEX), (low, lst.LST_EINDEX),
                      (high, lst.LST_EINDEX), (fine[::-1].copy(), lst.LST_EINDEX)):
        at = torch.tensor(off, dtype=torch.int32, device="cuda")
        _, _, saved = layer.forward(x, g, at, save=True)
        assert layer.sync() == code
        layer.backward(x, g, dy, saved, at)
        assert layer.sync() == code


@pytest.mark.gpu
@pytest.mark.parametrize("gate", [0.0, -3.0, -9.0])
def test_an_infinite_state_stays_in_its_sequence(gpu_lib, gate):
    """It is no finite number again before the sequence's end, and nothing else changes."""
    x, g, off, dy, h0, dlast = _inputs((40, 900, 70), 12, torch.float32, 23)
    g.add_(gate)
    at = torch.tensor(off, dtype=torch.int32, device="cuda")

    def both():
        y, last, saved = lst.lst_recur_forward(x, g, at, h0, save=True)
        return (y, last, *lst.lst_recur_backward(x, g, dy, saved, at, h0, dlast))

    want = both()
    x[45, 3] = float("inf")
    got = both()
    assert not got[0][45:940, 3].isfinite().any() and not got[1][1, 3].isfinite()
    assert not got[3][45:940, 3].isfinite().any()  # their gates' gradients
    for a in (got[0], want[0], got[3], want[3]):
        a[45:940, 3] = 0
    got[1][1, 3] = want[1][1, 3] = 0
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_shut_gates_of_any_type(gpu_lib, dtype):
    """Gates that let next to nothing in, or out: what does pass has float32's digits in the
    states, which are float32 whatever the rows' type."""
    n, d = 300, 64
    torch.manual_seed(31)
    size = torch.linspace(9, 85, d, device="cuda")
    x, dy = (torch.randn((n, d), device="cuda").to(dtype) for _ in range(2))
    for sign in (1.0, -1.0):
        g = (sign * size * (1 + 0.01 * torch.rand((n, d), device="cuda"))).to(dtype)
        for h0 in (None, torch.randn((1, d), device="cuda")):
            _check_all(x, g, np.array([0, n]), dy, h0, None)
            layer = lst.GatedRecurrence(d)
            h = torch.zeros((n, d), device="cuda")
            y = layer.step(x, g, h)
            off = np.arange(n + 1)
            wy, wl, ey, el, _ = between.recur(_np(x), _np(g), off)
            _check(y, wy, ey, dtype)
            _check(h, wl, el)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_gates_without_end_of_any_type(gpu_lib, dtype):
    """Infinite gates keep the state or take the row exactly, also the largest finite ones; a gate
    that is no number leaves none."""
    n, d = 200, 6
    torch.manual_seed(32)
    x = torch.randn((n, d), device="cuda").to(dtype)
    g = torch.zeros((n, d), device="cuda").to(dtype)
    big = torch.finfo(dtype).max
    g[:, 0], g[:, 1], g[:, 2], g[:, 3] = float("inf"), -float("inf"), big, -big
    g[90, 4] = float("nan")
    h0 = torch.randn((1, d), device="cuda")
    y, last, _ = lst.lst_recur_forward(x, g, None, h0)
    for c in (0, 2):
        assert torch.equal(y[:, c], h0[0, c].to(dtype).expand(n)) and last[0, c] == h0[0, c]
    for c in (1, 3):
        assert torch.equal(y[:, c], x[:, c])
    assert y[:90, 4].isfinite().all() and y[90:, 4].isnan().all() and last[0, 4].isnan()
    assert y[:, 5].isfinite().all()
    h = h0.repeat(n, 1)
    lst.lst_recur_step(x, g, h)
    assert torch.equal(h[:, 0], h0[0, 0].expand(n)) and torch.equal(h[:, 3], x[:, 3].float())
    assert h[90, 4].isnan() and h[:90, 4].isfinite().all()
