"""What a kept input costs a weight gradient, against the call on the tensor itself: no more than the format's error of every value."""
import pytest
import torch

from oracle import sparse_conv as oc
from workloads import generators as gen
from _rows import steps
from _util import coords_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("ci,co", [(16, 16), (40, 24), (64, 64)])
def test_weight_gradient(dtype, ci, co):
    """A value is off by half a step, or by less than one where it is beyond 127.5 steps or below half of one.  dW sums these with the
    magnitudes of dy; what else differs are two fp32 sums of n exact products (of 22 bits or, in fp32, rounded ones) each."""
    import paper_2311_12862_amd as sp
    coords = gen.lidar_scene(51, target_n=900)
    M = oc.build_kmap(coords, 3, 1).M
    km = sp.build_kmap(coords_dev(coords), 3, 1)
    g = torch.Generator(device="cuda").manual_seed(ci)
    x = torch.randn(km.n_in, ci, generator=g, device="cuda").relu().to(dtype)      # (a ReLU's output)
    d = torch.randn(km.n_out, co, generator=g, device="cuda").to(dtype)
    kept = sp.q8_pack(x)
    step = steps("cuda")[kept.exps.long()].repeat_interleave(32, 1)[:, :ci]
    size = x.double().abs() / step
    off = torch.where((size >= 0.5) & (size <= 127.5) | (size == 0), 0.5 * step * (size > 0), step)
    np64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    bound = torch.from_numpy(oc.wgrad(np64(off), np64(d.abs()), M))
    sums = torch.from_numpy(oc.wgrad(np64(x.abs() + off), np64(d.abs()), M)) * (2 * (km.n_out + 2) * 2.0 ** -24)
    diff = sp.wgrad(kept, d, km).double() - sp.wgrad(x, d, km).double()
    assert (diff.cpu().abs() <= bound + sums).all()
    assert diff.abs().max() > 0                  # (the checkpoint is what was read)
