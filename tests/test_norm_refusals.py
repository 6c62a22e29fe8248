"""What layer norm and the 8-bit checkpoints refuse: by the C ABI's status codes and by the binding's errors, no GPU needed."""
import ctypes as C

import pytest
import torch

import paper_2311_12862_amd as sp
from paper_2311_12862_amd.binding import Q8

P = C.c_void_p(4096)          # an address that no refused call looks at
OK, EINVAL = 0, -1


@pytest.fixture(scope="module")
def lib():
    return sp.load_library()


def _q8(data=4096, exps=4096):
    return C.byref(Q8(data, exps))


@pytest.mark.parametrize("rows,c,dtype", [(-1, 8, 1), (4, 0, 1), (4, -8, 1), (4, 4097, 1), (1 << 39, 4, 1), (4, 8, 3), (4, 8, -1)])
def test_sizes_and_types(lib, rows, c, dtype):
    assert lib.spconv_q8_pack(P, rows, c, dtype, _q8(), None) == EINVAL
    assert lib.spconv_q8_unpack(_q8(), rows, c, dtype, P, None) == EINVAL
    assert lib.spconv_layer_norm_fwd(P, None, None, None, 1e-5, 0, rows, c, dtype, P, P, None, None, None) == EINVAL
    assert lib.spconv_layer_norm_bwd(P, P, None, None, None, None, P, rows, c, dtype, P, None, P, P, P, 1 << 40, None) == EINVAL
    if dtype == 1:
        assert lib.spconv_layer_norm_bwd_workspace(rows, c) == EINVAL


def test_null_pointers(lib):
    assert lib.spconv_q8_pack(None, 4, 8, 1, _q8(), None) == EINVAL
    assert lib.spconv_q8_pack(P, 4, 8, 1, None, None) == EINVAL
    assert lib.spconv_q8_pack(P, 4, 8, 1, _q8(None), None) == EINVAL
    assert lib.spconv_q8_pack(P, 4, 8, 1, _q8(4096, None), None) == EINVAL
    assert lib.spconv_q8_unpack(None, 4, 8, 1, P, None) == EINVAL
    assert lib.spconv_q8_unpack(_q8(), 4, 8, 1, None, None) == EINVAL
    assert lib.spconv_q8_unpack(_q8(4096, None), 4, 8, 1, P, None) == EINVAL
    assert lib.spconv_relu_bwd_q8(None, _q8(), P, 8, 1, None) == EINVAL
    assert lib.spconv_relu_bwd_q8(P, None, P, 8, 1, None) == EINVAL
    assert lib.spconv_relu_bwd_q8(P, _q8(None), P, 8, 1, None) == EINVAL
    assert lib.spconv_relu_bwd_q8(P, _q8(), None, 8, 1, None) == EINVAL
    assert lib.spconv_relu_bwd_q8(P, _q8(), P, -1, 1, None) == EINVAL
    assert lib.spconv_relu_bwd_q8(P, _q8(), P, 8, 5, None) == EINVAL
    assert lib.spconv_wgrad_q8(None, P, None, 64, 64, 1, None, P, None) == EINVAL
    fwd = lambda **k: lib.spconv_layer_norm_fwd(  # noqa: E731
        k.get("x", P), None, None, None, k.get("eps", 1e-5), k.get("relu", 0), 4, 8, 1, k.get("y", P), P, k.get("kx"), k.get("ky"), None)
    assert fwd(x=None) == EINVAL and fwd(y=None) == EINVAL
    assert fwd(eps=-1e-6) == EINVAL and fwd(eps=float("nan")) == EINVAL and fwd(relu=2) == EINVAL and fwd(relu=-1) == EINVAL
    assert fwd(kx=_q8(), ky=_q8(4096, 8192)) == EINVAL and fwd(kx=_q8(), ky=_q8(8192, 4096)) == EINVAL   # one place for two
    assert fwd(kx=_q8(None)) == EINVAL and fwd(kx=_q8(4096, None)) == EINVAL and fwd(ky=_q8(None)) == EINVAL


def test_backward_arguments(lib):
    need = lib.spconv_layer_norm_bwd_workspace(4000, 8)
    assert need > 0 and lib.spconv_layer_norm_bwd_workspace(4, 8) == 0

    def bwd(dout=P, x=P, kx=None, y=None, ky=None, stats=P, dx=P, dw=P, db=P, ws=P, n=need):
        return lib.spconv_layer_norm_bwd(dout, x, kx, y, ky, None, stats, 4000, 8, 1, dx, None, dw, db, ws, n, None)

    assert bwd(dout=None) == EINVAL and bwd(x=None) == EINVAL and bwd(stats=None) == EINVAL and bwd(dx=None) == EINVAL
    assert bwd(kx=_q8()) == EINVAL                       # both inputs
    assert bwd(y=P, ky=_q8()) == EINVAL                  # both outputs
    assert bwd(x=None, kx=_q8(4096, None)) == EINVAL
    assert bwd(ky=_q8(None)) == EINVAL
    assert bwd(dw=None) == EINVAL and bwd(db=None) == EINVAL   # one of two
    assert bwd(ws=None) == EINVAL and bwd(n=need - 1) == EINVAL


def test_nothing_to_do(lib):
    assert lib.spconv_q8_pack(None, 0, 8, 1, _q8(None, None), None) == OK
    assert lib.spconv_q8_unpack(_q8(None, None), 0, 8, 1, None, None) == OK
    assert lib.spconv_relu_bwd_q8(None, _q8(None, None), None, 0, 1, None) == OK
    assert lib.spconv_layer_norm_fwd(None, None, None, None, 1e-5, 1, 0, 8, 1, None, None, None, None, None) == OK
    assert lib.spconv_layer_norm_bwd(None, None, None, None, None, None, None, 0, 8, 1, None, None, None, None, None, 0, None) == OK


def test_binding_takes_device_tensors_only():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        sp.q8_pack(x)
    with pytest.raises(ValueError):
        sp.layer_norm_fwd(x)
    with pytest.raises(ValueError):
        sp.layer_norm_bwd(x, x, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        sp.Checkpoint(torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        sp.Checkpoint.empty(4, 8, "cpu")
    with pytest.raises(ValueError):
        sp.Checkpoint.empty(4, 0)


@pytest.mark.gpu
def test_binding_checks_shapes_and_types():
    x = torch.zeros(4, 40, device="cuda")
    kept, other = sp.q8_pack(x), sp.Checkpoint.empty(4, 41)
    y, stats = sp.layer_norm_fwd(x)
    w = torch.ones(40, device="cuda")
    with pytest.raises(ValueError):
        sp.Checkpoint(kept.data, kept.exps[:, :1].contiguous())
    with pytest.raises(ValueError):
        sp.Checkpoint(kept.data, kept.data)
    with pytest.raises(ValueError):
        sp.q8_pack(x.double())
    with pytest.raises(ValueError):
        sp.q8_pack(x.t())
    with pytest.raises(ValueError):
        sp.q8_pack(x[0])
    with pytest.raises(ValueError):
        sp.q8_unpack(kept, torch.float64)
    with pytest.raises(ValueError):
        sp.ew(sp.EW_ADD, x, kept)
    with pytest.raises(ValueError):
        sp.ew(sp.EW_RELU_BWD, x[:3], kept)
    with pytest.raises(ValueError):
        sp.layer_norm_fwd(x, w.half())
    with pytest.raises(ValueError):
        sp.layer_norm_fwd(x, residual=x.half())
    with pytest.raises(ValueError):
        sp.layer_norm_bwd(x, None, stats)
    with pytest.raises(ValueError):
        sp.layer_norm_bwd(x, x.half(), stats)
    for call in (lambda: sp.q8_pack(x, other), lambda: sp.q8_unpack(kept, torch.float32, x[:3]), lambda: sp.layer_norm_fwd(x, w[:39]),
                 lambda: sp.layer_norm_fwd(x, keep_x=other), lambda: sp.layer_norm_fwd(x, keep_x=kept, keep_y=kept), lambda: sp.layer_norm_fwd(x, out=x[:3]), lambda: sp.layer_norm_fwd(x, eps=-1.0),
                 lambda: sp.layer_norm_bwd(x, other, stats), lambda: sp.layer_norm_bwd(x, x, stats, gate=other),
                 lambda: sp.layer_norm_bwd(x, x, stats[:3]), lambda: sp.layer_norm_bwd(x[:3], x, stats[:3])):
        with pytest.raises(sp.SpconvError):
            call()
    km = sp.build_kmap(torch.tensor([[0, i, 0, 0] for i in range(4)], dtype=torch.int32, device="cuda"), 3, 1)
    with pytest.raises(sp.SpconvError):
        sp.wgrad(sp.Checkpoint.empty(5, 40), x, km)
    with pytest.raises(sp.SpconvError):
        sp.wgrad(sp.Checkpoint.empty(4, 41), x, km)          # channels
    with pytest.raises(ValueError):
        sp.wgrad(kept, x.double(), km)
    assert torch.isfinite(y).all()
