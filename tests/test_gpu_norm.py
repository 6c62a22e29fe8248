"""Layer norm and its gradients against 64-bit forms, with tolerances from the number of fp32 operations (tests/_rows.py)."""
import pytest
import torch

from _rows import bwd64, fwd64, pack64, unpack64, within

pytestmark = pytest.mark.gpu
DTS = [torch.float32, torch.float16, torch.bfloat16]
WIDTHS = [1, 2, 7, 8, 16, 20, 31, 32, 33, 40, 45, 64, 96, 100, 256, 264, 513, 520, 1000, 2056, 4091, 4096]
EPS = 1e-5


def _rows(rows, c, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, c, generator=g, device="cuda") * (0.1 + 2 * torch.rand(rows, 1, generator=g, device="cuda"))
    x = x + 3 * torch.randn(rows, 1, generator=g, device="cuda")
    if rows > 4:
        x[1] = 0                # an empty voxel
        x[2] = 2.5              # no variance
        x[3] = 100 + 0.01 * x[3]  # an offset far above the spread
    return x.to(dtype)


def _params(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return 1 + 0.3 * torch.randn(c, generator=g, device="cuda"), 0.3 * torch.randn(c, generator=g, device="cuda")


def _shifted(t, shift):
    """The same values, `shift` elements past an aligned address, and the room around them."""
    room = torch.full((t.numel() + 16,), 7.0, dtype=t.dtype, device=t.device)
    view = room[shift:shift + t.numel()].view(t.shape)
    view.copy_(t)
    return view, room


def _check_fwd(rows, c, dtype, affine, relu, residual, shift=0, seed=0):
    import paper_2311_12862_amd as sp
    x, _ = _shifted(_rows(rows, c, dtype, seed + c), shift)
    w, b = _params(c, c) if affine else (None, None)
    res = _rows(rows, c, dtype, seed + 1) if residual else None
    out, room = _shifted(torch.zeros_like(x), shift)
    kept_x, kept_y = sp.Checkpoint.empty(rows, c), sp.Checkpoint.empty(rows, c)
    y, stats = sp.layer_norm_fwd(x, w, b, EPS, relu=relu, residual=res, out=out, keep_x=kept_x, keep_y=kept_y)
    want, want_stats, tol, tol_stats = fwd64(x, w, b, EPS, relu, res)
    within(y, want, tol, dtype)
    within(stats, want_stats, tol_stats)
    for kept, t in ((kept_x, x), (kept_y, y)):
        q, e = pack64(t)
        assert torch.equal(kept.data, q) and torch.equal(kept.exps, e)
    assert (room[shift + rows * c:] == 7).all() and (room[:shift] == 7).all()
    again, stats2 = sp.layer_norm_fwd(x, w, b, EPS, relu=relu, residual=res)     # without the checkpoints: the same bits
    assert torch.equal(again, y) and torch.equal(stats, stats2)


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("c", WIDTHS)
def test_forward(dtype, c):
    _check_fwd(37, c, dtype, True, True, True)
    _check_fwd(1, c, dtype, True, False, False)


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("affine,relu,residual", [(False, False, False), (False, True, True), (True, True, False), (True, False, True)])
def test_forward_variants(dtype, affine, relu, residual):
    for rows, c, shift in ((1000, 64, 0), (333, 64, 1), (257, 45, 3)):
        _check_fwd(rows, c, dtype, affine, relu, residual, shift)


def _check_bwd(rows, c, dtype, affine, relu, residual, kept, shift=0, grads=True):
    import paper_2311_12862_amd as sp
    x, _ = _shifted(_rows(rows, c, dtype, c), shift)
    w, b = _params(c, c) if affine else (None, None)
    y, stats = sp.layer_norm_fwd(x, w, b, EPS, relu=relu)
    if relu and rows > 5:
        y[4] = 0                                   # a row that nothing goes through
    dout = _rows(rows, c, dtype, c + 1)
    values, gate = x, (y > 0 if relu else None)
    use_x, use_y = x, (y if relu else None)
    if kept >= 1:
        use_x = sp.q8_pack(x)
        values = unpack64(use_x.data, use_x.exps)
    if kept >= 2 and relu:
        use_y = sp.q8_pack(y)
    dx, dw, db, dres = sp.layer_norm_bwd(dout, use_x, stats, w, gate=use_y, residual=residual, affine=grads)
    want, tol = bwd64(dout, values, stats, w, gate)
    within(dx, want[0], tol[0], dtype)
    if grads:
        within(dw, want[1], tol[1])
        within(db, want[2], tol[2])
    else:
        assert dw is None and db is None
    if residual:
        assert torch.equal(dres.double(), want[3])
    else:
        assert dres is None
    if relu and rows > 5:
        assert (dx[4] == 0).all()
    again = sp.layer_norm_bwd(dout, use_x, stats, w, gate=use_y, residual=residual, affine=grads)
    assert torch.equal(dx, again[0]) and (not grads or (torch.equal(dw, again[1]) and torch.equal(db, again[2])))


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("kept", [0, 2])
def test_backward(dtype, c, kept):
    _check_bwd(37, c, dtype, True, True, True, kept)
    _check_bwd(1, c, dtype, True, False, False, kept)


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("affine,relu,residual,kept,grads", [(False, False, False, 0, True), (True, True, False, 1, True),
                                                             (True, False, True, 1, False), (False, True, True, 2, False)])
def test_backward_variants(dtype, affine, relu, residual, kept, grads):
    for rows, c, shift in ((1000, 64, 0), (333, 64, 1), (257, 45, 3), (9001, 256, 0)):
        _check_bwd(rows, c, dtype, affine, relu, residual, kept, shift, grads)


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("rows,c", [(512, 32), (513, 32), (128, 100), (129, 100), (4, 4096), (5, 4096), (512, 8), (513, 3)])
def test_backward_around_one_workgroup(dtype, rows, c):
    """As many rows as one workgroup takes alone, and one more."""
    for kept in (0, 2):
        _check_bwd(rows, c, dtype, True, True, True, kept)


@pytest.mark.parametrize("dtype,c", [(torch.float16, 32), (torch.bfloat16, 256), (torch.float32, 45)])
def test_many_rows(dtype, c):
    _check_fwd(150_001, c, dtype, True, True, True)
    _check_bwd(150_001, c, dtype, True, True, True, 2)


def test_gradients_against_differences():
    """fp32 gradients against central differences of the 64-bit forward form, no element near the ReLU's corner."""
    import paper_2311_12862_amd as sp
    rows, c, h = 3, 10, 1e-5
    x, res = _rows(rows, c, torch.float32, 11), _rows(rows, c, torch.float32, 12)
    w, b = _params(c, 13)
    dout = _rows(rows, c, torch.float32, 14)
    y, stats = sp.layer_norm_fwd(x, w, b, EPS, relu=True, residual=res)
    pre = fwd64(x, w, b, EPS, False, res)[0]
    assert pre.abs().min() > 1e-3
    dx, dw, db, dres = sp.layer_norm_bwd(dout, x, stats, w, gate=y, residual=True)
    loss = lambda *a: (fwd64(a[0], a[1], a[2], EPS, True, a[3])[0] * dout.double()).sum()  # noqa: E731
    at = [x.double(), w.double(), b.double(), res.double()]
    for i, got in enumerate((dx, dw, db, dres)):
        want = torch.empty_like(at[i])
        for e in range(at[i].numel()):
            low, high = [t.clone() for t in at], [t.clone() for t in at]
            low[i].view(-1)[e] -= h
            high[i].view(-1)[e] += h
            want.view(-1)[e] = (loss(*high) - loss(*low)) / (2 * h)
        # differences: h^2 of the third derivative (below 1e3 here) and 2^-53 / h of the loss; the kernel: a few hundred roundings of
        # values below the scale
        scale = max(1.0, want.abs().max().item())
        assert (got.double() - want).abs().max().item() <= 1e-6 * scale + 300 * 2 ** -24 * scale * 10, i


@pytest.mark.parametrize("dtype", DTS)
def test_rows_that_are_not_finite_stay_their_own(dtype):
    import paper_2311_12862_amd as sp
    x = _rows(70, 64, dtype, 3)
    w, b = _params(64, 3)
    good, good_stats = sp.layer_norm_fwd(x, w, b, relu=True)
    x[9, 3], x[20, 60], x[33, 0] = float("inf"), float("nan"), float("-inf")
    kept_x, kept_y = sp.Checkpoint.empty(70, 64), sp.Checkpoint.empty(70, 64)
    y, stats = sp.layer_norm_fwd(x, w, b, relu=True, keep_x=kept_x, keep_y=kept_y)
    bad = torch.tensor([9, 20, 33], device="cuda")
    fine = torch.ones(70, dtype=torch.bool, device="cuda")
    fine[bad] = False
    assert torch.equal(y[fine], good[fine]) and torch.equal(stats[fine], good_stats[fine])
    assert torch.isnan(y[bad]).all()                       # a ReLU does not hide them
    q, e = pack64(x)
    assert torch.equal(kept_x.data, q) and torch.equal(kept_x.exps, e)
    q, e = pack64(y)
    assert torch.equal(kept_y.data, q) and torch.equal(kept_y.exps, e)
    dx = sp.layer_norm_bwd(torch.ones_like(x), x, stats, w, gate=y)[0]
    want = sp.layer_norm_bwd(torch.ones_like(x), x, good_stats, w, gate=good)[0]
    assert torch.equal(dx[fine], want[fine]) and torch.isnan(dx[bad]).all()


def test_no_rows():
    import paper_2311_12862_amd as sp
    x = torch.empty(0, 48, device="cuda")
    y, stats = sp.layer_norm_fwd(x)
    assert y.shape == (0, 48) and stats.shape == (0, 2)
    dx, dw, db, dres = sp.layer_norm_bwd(x, x, stats, residual=True)
    assert dx.shape == (0, 48) and dres.shape == (0, 48) and (dw == 0).all() and (db == 0).all() and dw.shape == (48,)


def test_in_place():
    import paper_2311_12862_amd as sp
    x, res = _rows(301, 96, torch.bfloat16, 1), _rows(301, 96, torch.bfloat16, 2)
    w, b = _params(96, 3)
    want, _ = sp.layer_norm_fwd(x, w, b, relu=True, residual=res)
    for out in ("x", "res"):
        a, r = x.clone(), res.clone()
        sp.layer_norm_fwd(a, w, b, relu=True, residual=r, out=a if out == "x" else r)
        assert torch.equal(a if out == "x" else r, want)


def test_offsets_beyond_32_bits():
    import paper_2311_12862_amd as sp
    rows, c, n = 48_000_011, 48, 2000                        # 2.3e9 elements
    x = torch.zeros(rows, c, dtype=torch.bfloat16, device="cuda")
    x[-n:] = _rows(n, c, torch.bfloat16, 4)
    w, b = _params(c, 5)
    kept = sp.Checkpoint.empty(rows, c)
    y, stats = sp.layer_norm_fwd(x, w, b, keep_x=kept)
    want, _, tol, _ = fwd64(x[-n:], w, b, EPS, False, None)
    within(y[-n:], want, tol, torch.bfloat16)
    dout = torch.zeros_like(x)
    dout[-n:] = _rows(n, c, torch.bfloat16, 6)
    dx, dw, db, _ = sp.layer_norm_bwd(dout, kept, stats, w, gate=y)
    values = unpack64(kept.data[-n:], kept.exps[-n:])
    want, tol = bwd64(dout[-n:], values, stats[-n:], w, y[-n:] > 0)
    within(dx[-n:], want[0], tol[0], torch.bfloat16)
    within(dw, want[1], tol[1])
    within(db, want[2], tol[2])


def test_on_another_stream():
    """All work on the caller's stream, between that stream's other work; the call's workspace outlives the call."""
    import paper_2311_12862_amd as sp
    x0, dout0 = _rows(60_001, 64, torch.float16, 1), _rows(60_001, 64, torch.float16, 2)
    w, b = _params(64, 3)
    y0, stats0 = sp.layer_norm_fwd(x0, w, b, relu=True)
    want = sp.layer_norm_bwd(dout0, x0, stats0, w, gate=y0, residual=True)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        x, dout = torch.zeros_like(x0), torch.zeros_like(dout0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            x.copy_(x0)
            dout.copy_(dout0)
        kept = sp.Checkpoint.empty(*x.shape)
        y, stats = sp.layer_norm_fwd(x, w, b, relu=True, keep_y=kept, stream=stream)
        got = sp.layer_norm_bwd(dout, x, stats, w, gate=kept, residual=True, stream=stream)
        junk = [torch.full((1 << 21,), 1.0, device="cuda") for _ in range(8)]      # would land in a workspace given back early
        side.synchronize()
        assert torch.equal(y, y0) and all(torch.equal(a, b2) for a, b2 in zip(got, want))
        del junk


def test_replays_in_a_hip_graph():
    """Forward with both checkpoints and backward from them, captured once, replayed on new inputs with eager work in between;
    a second graph of the same call lives beside it."""
    import paper_2311_12862_amd as sp
    shape = (20_011, 96)
    w, b = _params(96, 3)
    x, res, dout = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(3))

    def step(x, res, dout):
        kept_x, kept_y = sp.Checkpoint.empty(*shape), sp.Checkpoint.empty(*shape)
        y, stats = sp.layer_norm_fwd(x, w, b, relu=True, residual=res, keep_x=kept_x, keep_y=kept_y)
        grads = sp.layer_norm_bwd(dout, kept_x, stats, w, gate=kept_y, residual=True)
        return (y, stats, sp.ew(sp.EW_RELU_BWD, dout, kept_y), sp.q8_unpack(sp.q8_pack(y), torch.bfloat16), *grads)

    for t in (x, res, dout):
        t.copy_(_rows(*shape, torch.bfloat16, 1))
    step(x, res, dout)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = step(x, res, dout)
        graphs.append((g, outs))
    for replay in range(4):
        for i, t in enumerate((x, res, dout)):
            t.copy_(_rows(*shape, torch.bfloat16, 10 * replay + i))
        want = [t.clone() for t in step(x, res, dout)]
        for g, outs in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, outs in graphs:
            assert all(torch.equal(a, c) for a, c in zip(outs, want)), replay


@pytest.mark.parametrize("c", [5, 45, 96, 600, 2050])
def test_backward_in_place(c):
    """The C call lets dx be dout."""
    import ctypes as C

    import paper_2311_12862_amd as sp
    x, dout = _rows(203, c, torch.float16, 1), _rows(203, c, torch.float16, 2)   # (one workgroup at c = 5 and 45)
    w, b = _params(c, 3)
    y, stats = sp.layer_norm_fwd(x, w, b, relu=True)
    want = sp.layer_norm_bwd(dout, x, stats, w, gate=y)
    lib = sp.load_library()
    ws = torch.empty(lib.spconv_layer_norm_bwd_workspace(203, c), dtype=torch.int8, device="cuda")
    dw, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib.spconv_layer_norm_bwd(p(dout), p(x), None, p(y), None, p(w), p(stats), 203, c, 1, p(dout), None, p(dw), p(db), p(ws),
                                     ws.numel(), stream) == 0
    assert torch.equal(dout, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])


def test_two_threads_on_two_streams():
    import threading

    import paper_2311_12862_amd as sp
    inputs = [(_rows(30_001, 64, torch.float16, s), _rows(30_001, 64, torch.float16, s + 10)) for s in range(2)]
    w, b = _params(64, 3)

    def step(x, dout):
        kept = sp.Checkpoint.empty(*x.shape)
        y, stats = sp.layer_norm_fwd(x, w, b, relu=True, keep_x=kept)
        return (y, *sp.layer_norm_bwd(dout, kept, stats, w, gate=y, residual=True))

    want = [step(*i) for i in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(40):
                got = step(*inputs[k])
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, c) for a, c in zip(got, want[k])):
                    wrong.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_one_of_weight_and_bias_and_no_statistics():
    """Weights at odd addresses, one of the two alone, and the C call without statistics."""
    import ctypes as C

    import paper_2311_12862_amd as sp
    for c in (45, 64):
        x = _rows(100, c, torch.float16, c)
        w, b = (_shifted(t, 1 + i)[0] for i, t in enumerate(_params(c, 7)))
        for weight, bias in ((w, None), (None, b), (w, b)):
            y, stats = sp.layer_norm_fwd(x, weight, bias, EPS)
            want, _, tol, _ = fwd64(x, weight, bias, EPS, False, None)
            within(y, want, tol, torch.float16)
        p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
        got = torch.empty_like(y)
        assert sp.load_library().spconv_layer_norm_fwd(p(x), None, p(w), p(b), EPS, 0, 100, c, 1, p(got), None, None, None,
                                                       C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        assert torch.equal(got, y)
        dout = _rows(100, c, torch.float16, 9)
        values, tol = bwd64(dout, x, stats, w, None)
        within(sp.layer_norm_bwd(dout, x, stats, w)[0], values[0], tol[0], torch.float16)


def test_eps_of_zero_and_a_large_one():
    """A row without variance has y = bias, not a NaN."""
    import paper_2311_12862_amd as sp
    x = torch.zeros(9, 40, device="cuda")
    x[4:] = _rows(5, 40, torch.float32, 1)
    w, b = _params(40, 2)
    y, stats = sp.layer_norm_fwd(x, w, b, 0.0)
    assert torch.isfinite(y).all() and torch.equal(y[:4], b.expand(4, 40))
    dx, dw, db, _ = sp.layer_norm_bwd(torch.zeros_like(x), x, stats, w)
    assert (dx == 0).all() and (dw == 0).all() and (db == 0).all()
    y, _ = sp.layer_norm_fwd(x, w, b, 1e30)
    assert (y - b).abs().max().item() < 1e-12 + 2 ** -24 * b.abs().max().item()


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("first", [9, 33, 129, 521])
def test_every_end_of_a_row(dtype, first):
    """Widths that leave 0 to 7 elements behind the last whole vector, rows at odd addresses, in a group of lanes of each kind."""
    for c in range(first, first + 8):
        for rows in (1, 67):
            _check_fwd(rows, c, dtype, True, True, True, shift=c % 3)
            _check_bwd(rows, c, dtype, True, True, True, 2 * (c % 2), shift=c % 3)
