"""8-bit checkpoints against the format's definition in 64 bits, bit for bit, and the readers of kept activations."""
import numpy as np
import pytest
import torch

from oracle import sparse_conv as oc
from workloads import generators as gen
from _rows import pack64, steps, unpack64
from _util import coords_dev, norm_err

pytestmark = pytest.mark.gpu
DTS = [torch.float32, torch.float16, torch.bfloat16]
WIDTHS = [1, 2, 7, 8, 16, 20, 31, 32, 33, 40, 45, 64, 96, 100, 256, 520, 4096]


def _values(rows, c, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, c, generator=g, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda"))
    return x.to(dtype)


def _same(kept, want):
    assert torch.equal(kept.exps, want[1])
    assert torch.equal(kept.data, want[0])


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("shift", [0, 1])
def test_pack_and_unpack(dtype, c, shift):
    import paper_2311_12862_amd as sp
    for rows in (1, 3, 130):
        x = _values(rows * c + shift, 1, dtype, c + rows)[shift:].view(rows, c)
        q, b = pack64(x)
        kept = sp.q8_pack(x)
        _same(kept, (q, b))
        room = torch.full((rows * c + 2,), 7.0, dtype=dtype, device="cuda")
        out = sp.q8_unpack(kept, dtype, room[shift:shift + rows * c].view(rows, c))
        assert torch.equal(out.double(), unpack64(q, b))        # exact: nothing is rounded
        assert (room[shift + rows * c:] == 7).all() and (not shift or room[0] == 7)


@pytest.mark.parametrize("dtype", DTS)
def test_special_values(dtype):
    """Zeros, ties, the type's ends, subnormals, infinities, NaN, and values that would round to 0 or to 128."""
    import paper_2311_12862_amd as sp
    top, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    sub = tiny * torch.finfo(dtype).eps
    rows = [[0.0, -0.0, 0.0], [1.0, 0.0078125, -0.0078125], [1.0, 0.0234375, -0.0390625], [1.0, 0.001, -0.001],
            [1.9921875, -1.9921875, 0.0], [top, -top, tiny], [tiny, sub, -sub], [sub, -sub, 0.0], [tiny, top, -sub],
            [float("inf"), 1.0, -1.0], [1.0, float("nan"), -1.0], [float("-inf"), float("nan"), 0.0], [127.5, 127.75, -127.99]]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype).cuda()
    x = torch.cat([x, x.flip(1), torch.zeros(len(rows), 29, dtype=dtype, device="cuda"), x * 0.5], 1)   # 38 channels, two blocks
    q, b = pack64(x)
    kept = sp.q8_pack(x)
    _same(kept, (q, b))
    assert torch.equal(torch.sign(kept.data.float())[torch.isfinite(x).all(1)], torch.sign(x.float())[torch.isfinite(x).all(1)])
    for out in DTS:
        got, want = sp.q8_unpack(kept, out).double(), unpack64(q, b)
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan)
        # in its own type a checkpoint's values are exact; another type's range may end before
        fits = ~nan & (want.to(out).double() == want)
        assert torch.equal(got[fits], want[fits])
        assert fits[~nan].all() or out != dtype


def test_half_a_step():
    """A value is off by at most half a step, 2^-7 of the block's largest; kept signs and values beyond 127.5 steps by less than one."""
    import paper_2311_12862_amd as sp
    x = _values(4000, 96, torch.float32, 5)
    kept = sp.q8_pack(x)
    step = steps(x.device)[kept.exps.long()].repeat_interleave(32, 1)
    off, size = (sp.q8_unpack(kept, torch.float32).double() - x.double()).abs() / step, x.double().abs() / step
    plain = (size >= 0.5) & (size <= 127.5)
    assert (off[plain] <= 0.5).all() and (off < 1).all()


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("rows,c", [(1, 1), (3, 8), (7, 45), (130, 32), (1000, 100)])
def test_relu_gradient(dtype, rows, c):
    """Exactly the gradient by the output itself: a checkpoint keeps every sign."""
    import paper_2311_12862_amd as sp
    y = (_values(rows, c, dtype, 1).relu() * torch.logspace(-6, 0, c, device="cuda")).to(dtype)
    for shift in (0, 1):
        d = _values(rows * c + shift, 1, dtype, 2)[shift:].view(rows, c)
        want = sp.ew(sp.EW_RELU_BWD, d, y)
        kept = sp.q8_pack(y)
        assert torch.equal(sp.ew(sp.EW_RELU_BWD, d, kept), want)
        sp.ew(sp.EW_RELU_BWD, d, kept, d)    # in place
        assert torch.equal(d, want)


def test_nothing_gets_past_a_block_that_is_not_finite():
    import paper_2311_12862_amd as sp
    y = torch.ones(2, 64, device="cuda")
    y[1, 3] = float("inf")
    d = torch.ones(2, 64, device="cuda")
    got = sp.ew(sp.EW_RELU_BWD, d, sp.q8_pack(y))
    assert (got[0] == 1).all() and (got[1, :32] == 0).all() and (got[1, 32:] == 1).all()


def _map(kind, n=1200):
    import paper_2311_12862_amd as sp
    c = coords_dev(gen.lidar_scene(51, target_n=n))
    if kind == "sub3":
        return sp.build_kmap(c, 3, 1)
    if kind == "sub5":
        return sp.build_kmap(c, 5, 1)
    if kind == "one":
        return sp.build_kmap(c, 1, 1)
    if kind == "down":
        return sp.build_kmap(c, 3, 2)
    if kind == "down2":
        return sp.build_kmap(c, 2, 2)
    if kind == "up":
        return sp.build_kmap(c, 3, 2, transposed=True)
    if kind == "dense":       # many pairs a row: straight from the map for narrow layers
        return sp.build_kmap(coords_dev(gen.full_grid(40, 1, seed=3)), 3, 1)
    return sp.build_kmap(c, 3, 1, dilate=True)


def _wgrad(km, dtype, ci, co, cfg=None, seed=3):
    import paper_2311_12862_amd as sp
    x, d = _values(km.n_in, ci, dtype, seed), torch.randn(km.n_out, co, device="cuda").to(dtype)
    x[::17] = 0
    kept = sp.q8_pack(x)
    got = sp.wgrad(kept, d, km, cfg)
    values = sp.q8_unpack(kept, torch.float32)
    M = km.export().cpu().numpy() if km.K != 5 else km.export().cpu().numpy()
    want = oc.wgrad(values.cpu().numpy(), d.float().cpu().numpy(), M)
    assert norm_err(got, want) <= 1e-4     # fp32 sums of exact products, as for the tensor itself
    assert torch.equal(got, sp.wgrad(kept, d, km, cfg))
    return got


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("kind", ["sub3", "sub5", "one", "down", "down2", "up", "dilated"])
def test_wgrad_on_every_map(kind, dtype):
    _wgrad(_map(kind), dtype, 40, 24)


@pytest.mark.parametrize("ci,co", [(8, 16), (32, 32), (40, 64), (64, 24), (72, 96), (104, 40), (128, 136), (264, 16), (16, 264)])
@pytest.mark.parametrize("dtype", DTS)
def test_wgrad_channels(ci, co, dtype):
    import paper_2311_12862_amd as sp
    km = _map("sub3")
    for pieces in (0, 1, 33, 4000):
        _wgrad(km, dtype, ci, co, sp.Config(wgrad_pairs=pieces) if pieces else None, seed=ci)


@pytest.mark.parametrize("dtype,ci,co", [(torch.float16, 32, 32), (torch.bfloat16, 16, 32), (torch.bfloat16, 136, 200), (torch.float16, 256, 64)])
def test_wgrad_on_a_dense_map(dtype, ci, co):
    _wgrad(_map("dense"), dtype, ci, co)


@pytest.mark.parametrize("n", [1, 2, 33])
def test_wgrad_few_rows(n):
    import paper_2311_12862_amd as sp
    km = sp.build_kmap(coords_dev(gen.uniform_cloud(n, 4, seed=n)), 3, 1)
    for dtype in DTS:
        _wgrad(km, dtype, 64, 64)


def test_wgrad_of_a_block_that_is_not_finite():
    import paper_2311_12862_amd as sp
    km = _map("sub3")
    x, d = _values(km.n_in, 64, torch.float16, 1), torch.ones(km.n_out, 64, dtype=torch.float16, device="cuda")
    x[5, 40] = float("inf")
    dw = sp.wgrad(sp.q8_pack(x), d, km)
    centre = dw[13]
    assert torch.isfinite(centre[:32]).all() and torch.isnan(centre[32:]).all()


def test_wgrad_on_an_asynchronous_build_and_on_no_rows():
    import paper_2311_12862_amd as sp
    c = coords_dev(gen.lidar_scene(8, target_n=900))
    km = sp.build_kmap(c, 3, 1, asynchronous=True)
    _wgrad(km, torch.float16, 64, 64)
    km.status()
    none = sp.build_kmap(c[:0], 3, 1)
    dw = sp.wgrad(sp.Checkpoint.empty(0, 16), torch.empty(0, 8, device="cuda"), none)
    assert dw.shape == (27, 16, 8) and (dw == 0).all()


def test_no_rows():
    import paper_2311_12862_amd as sp
    kept = sp.q8_pack(torch.empty(0, 40, device="cuda"))
    assert kept.data.shape == (0, 40) and kept.exps.shape == (0, 2)
    assert sp.q8_unpack(kept, torch.float16).shape == (0, 40)
    assert sp.ew(sp.EW_RELU_BWD, torch.empty(0, 40, device="cuda"), kept).shape == (0, 40)


def test_offsets_beyond_32_bits():
    import paper_2311_12862_amd as sp
    rows, c = 48_000_011, 48                                   # 2.3e9 elements
    x = torch.zeros(rows, c, dtype=torch.bfloat16, device="cuda")
    x[-3000:] = _values(3000, c, torch.bfloat16, 4)
    kept = sp.q8_pack(x)
    q, b = pack64(x[-3000:])
    assert torch.equal(kept.data[-3000:], q) and torch.equal(kept.exps[-3000:], b)
    assert not kept.data[:-3000].any()
    out = sp.q8_unpack(kept, torch.bfloat16, x)
    assert torch.equal(out[-3000:].double(), unpack64(q, b))
    assert torch.equal(sp.ew(sp.EW_RELU_BWD, out, kept)[-3000:], out[-3000:].relu())


@pytest.mark.parametrize("ci,co", [(8, 16), (16, 16), (24, 8), (32, 32), (40, 64), (48, 64), (64, 64), (72, 96), (96, 96), (80, 40),
                                   (104, 128), (112, 128), (200, 136), (256, 256), (264, 200), (400, 72)])
@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("kind", ["sub3", "down", "dense"])
def test_wgrad_has_the_bits_of_the_unpacked_tensor(ci, co, dtype, kind):
    """The values are exact in every type and the sums' order is the tensor's."""
    import paper_2311_12862_amd as sp
    km = _map(kind)
    x = _values(km.n_in, ci, dtype, 9)
    x[3] = 0
    kept, d = sp.q8_pack(x), _values(km.n_out, co, dtype, 10)
    for pieces in (0, 1, 33, 4000) if kind == "sub3" else (0,):
        cfg = sp.Config(wgrad_pairs=pieces) if pieces else None
        assert torch.equal(sp.wgrad(kept, d, km, cfg), sp.wgrad(sp.q8_unpack(kept, dtype), d, km, cfg)), pieces


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_wgrad_of_every_exponent(dtype):
    """Blocks of every size that the type has, subnormal ones among them, and a checkpoint whose data stands at an odd address."""
    import paper_2311_12862_amd as sp
    km = _map("one", 700)
    low, high = (-24, 15) if dtype == torch.float16 else (-133, 127)
    x = torch.randn(km.n_in, 64, device="cuda", dtype=torch.float64).clamp(-1, 1)
    x = (x * torch.tensor([2.0 ** (low + i % (high - low + 1)) for i in range(km.n_in)], device="cuda", dtype=torch.float64)[:, None]).to(dtype)
    d = torch.zeros(km.n_out, 64, dtype=dtype, device="cuda")
    kept = sp.q8_pack(x)
    room = torch.zeros(km.n_in * 64 + 1, dtype=torch.int8, device="cuda")
    room[1:] = kept.data.flatten()
    odd = sp.Checkpoint(room[1:].view(km.n_in, 64), kept.exps)
    for row in range(0, km.n_in, 41):       # one row at a time: every value of it comes out as it is
        d.zero_()
        d[row, 5] = 1
        want = unpack64(kept.data[row:row + 1], kept.exps[row:row + 1])[0]
        for c in (kept, odd):
            assert torch.equal(sp.wgrad(c, d, km)[0, :, 5].double(), want), row


def test_wgrad_captured_then_a_larger_layer():
    """A captured call that unpacks replays on its own room after a wider layer of the kmap took a larger one."""
    import paper_2311_12862_amd as sp
    km, other = _map("sub3"), _map("sub3", 1500)
    x, d = _values(km.n_in, 24, torch.float32, 1), _values(km.n_out, 16, torch.float32, 2)
    kept = sp.q8_pack(x)
    sp.wgrad(kept, d, km)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sp.wgrad(kept, d, km)
    for replay in range(3):
        sp.q8_pack(_values(km.n_in, 24, torch.float32, 10 + replay), kept)
        want = sp.wgrad(kept, d, km).clone()
        wide = sp.wgrad(sp.q8_pack(_values(km.n_in, 40 + 8 * replay, torch.float32, 3)), _values(km.n_out, 64, torch.float32, 4), km)
        small = sp.wgrad(sp.q8_pack(_values(other.n_in, 24, torch.float32, 5)), _values(other.n_out, 16, torch.float32, 6), other)
        assert torch.isfinite(wide).all()
        before = small.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(small, before)


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("rows,c", [(3, 7), (70, 45), (33, 64), (5, 1000)])
def test_nothing_beside_a_checkpoint_is_written(dtype, rows, c):
    import paper_2311_12862_amd as sp
    nb = -(-c // 32)
    for shift in (0, 1, 3, 4):
        data = torch.full((rows * c + 16,), 99, dtype=torch.int8, device="cuda")
        exps = torch.full((rows * nb + 16,), 99, dtype=torch.uint8, device="cuda")
        kept = sp.Checkpoint(data[shift:shift + rows * c].view(rows, c), exps[shift:shift + rows * nb].view(rows, nb))
        x = _values(rows, c, dtype, c)
        sp.q8_pack(x, kept)
        q, b = pack64(x)
        _same(kept, (q, b))
        again = sp.Checkpoint(data[shift:shift + rows * c].view(rows, c).zero_(), kept.exps.zero_())
        sp.layer_norm_fwd(x, keep_x=again)
        _same(again, (q, b))
        for t, n in ((data, rows * c), (exps, rows * nb)):
            assert (t[:shift] == 99).all() and (t[shift + n:] == 99).all()
        assert torch.equal(sp.q8_unpack(kept, dtype).double(), unpack64(q, b))


@pytest.mark.parametrize("dtype", DTS)
def test_checkpoints_that_no_tensor_has(dtype):
    """Any bytes are a checkpoint: q = -128, steps of every size, b = 255 a NaN whatever q is; every reader sees the same values."""
    import paper_2311_12862_amd as sp
    km = _map("one", 600)
    n = km.n_in
    g = torch.Generator(device="cuda").manual_seed(1)
    data = torch.randint(-128, 128, (n, 64), generator=g, device="cuda").to(torch.int8)
    exps = torch.randint(100, 140, (n, 2), generator=g, device="cuda").to(torch.uint8)
    exps[7, 0] = 255
    exps[9, 1] = 0
    kept = sp.Checkpoint(data, exps)
    want = unpack64(data, exps)
    values = sp.q8_unpack(kept, dtype)
    assert torch.isnan(values[7, :32]).all() and torch.equal(torch.isnan(values), torch.isnan(want))
    within = ~torch.isnan(want) & (want.to(dtype).double() == want)
    assert torch.equal(values.double()[within], want[within])
    d = torch.zeros(n, 16, dtype=dtype, device="cuda")
    d[11, 3], d[9, 4], d[30, 5] = 1, 1, 1
    dw = sp.wgrad(kept, d, km)[0]
    rows = torch.tensor([11, 9, 30], device="cuda")
    got, fits = dw[:, 3:6].t().double(), within[rows]
    # (a NaN times a zero is a NaN: channels of the block that has one)
    assert torch.isnan(got[:, :32]).all() and torch.equal(got[:, 32:][fits[:, 32:]], want[rows][:, 32:][fits[:, 32:]])
