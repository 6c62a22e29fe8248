"""A checkpoint has no type of its own: what a reader of one type sees is q * 2^(b - 133) rounded to that type, whichever exponents the
block has, and whichever way the reader takes the values."""
import pytest
import torch

from workloads import generators as gen
from _util import coords_dev

pytestmark = pytest.mark.gpu


def _same(a, b):
    """Equal, NaN where the other is."""
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0)) and torch.equal(torch.isnan(a), torch.isnan(b))


def _points(n):
    import paper_2311_12862_amd as sp
    return sp.build_kmap(coords_dev(gen.uniform_cloud(n, 12, seed=1)), 1, 1)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("c", [32, 64, 96, 128, 256])
def test_every_exponent_and_byte(dtype, c):
    """One row that is not zero: column 5 of dW is that row as the reader saw it (products with 1, sums with 0)."""
    import paper_2311_12862_amd as sp
    km = _points(37)
    n, nb = km.n_in, c // 32
    data = torch.zeros((n, c), dtype=torch.int8, device="cuda")
    exps = torch.ones((n, nb), dtype=torch.uint8, device="cuda")
    d = torch.zeros((n, 16), dtype=dtype, device="cuda")
    d[7, 5] = 1
    kept = sp.Checkpoint(data, exps)
    bytes32 = (torch.arange(256, device="cuda") - 128).to(torch.int8).view(8, 32)
    bs = list(range(0, 5)) + list(range(60, 90, 7)) + list(range(95, 111)) + list(range(138, 152)) + [180, 200, 253, 254]
    calls = 0
    for part in range(8):                       # every byte meets every exponent
        for first in range(0, len(bs), nb):
            some = bs[first:first + nb]
            for j in range(nb):
                data[7, 32 * j:32 * j + 32] = bytes32[(part + j) % 8]
                exps[7, j] = some[j] if j < len(some) else 127
            got = sp.wgrad(kept, d, km)[0, :, 5]
            want = sp.q8_unpack(kept, dtype)[7].float()
            assert _same(got, want), (some, part)
            calls += 1
    assert calls >= 8


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("ci,co", [(32, 32), (40, 64), (96, 96), (128, 64), (256, 32)])
def test_checkpoints_of_fp32_tensors(dtype, ci, co):
    """Packed from fp32 with magnitudes around both ends of fp16: the bits of the call on the unpacked tensor."""
    import paper_2311_12862_amd as sp
    km = sp.build_kmap(coords_dev(gen.lidar_scene(51, target_n=900)), 3, 1)
    g = torch.Generator(device="cuda").manual_seed(ci)
    for low, high in ((-31, -17), (-8, 8), (9, 16), (13, 23)):
        ex = torch.randint(low, high + 1, (km.n_in, 1), generator=g, device="cuda").double()
        x = (torch.randn(km.n_in, ci, generator=g, device="cuda").double() * 2.0 ** ex).float()
        x[torch.rand(x.shape, generator=g, device="cuda") < 0.3] = 0
        kept = sp.q8_pack(x)
        d = torch.randn(km.n_out, co, generator=g, device="cuda").to(dtype)
        got, want = sp.wgrad(kept, d, km), sp.wgrad(sp.q8_unpack(kept, dtype), d, km)
        assert _same(got, want), (low, high)
        if dtype == torch.bfloat16 or high <= 8:
            assert torch.isfinite(got).all()


def test_the_address_does_not_decide():
    """Data at an odd address is unpacked first: the same answer."""
    import paper_2311_12862_amd as sp
    km = _points(300)
    x = torch.zeros((300, 64), device="cuda")
    x[:, ::3] = 100.0
    x[:, 32] = 70000.0                          # the block's step is 2^10: its other values stay numbers in fp16
    kept = sp.q8_pack(x)
    room = torch.zeros(300 * 64 + 1, dtype=torch.int8, device="cuda")
    room[1:] = kept.data.flatten()
    odd = sp.Checkpoint(room[1:].view(300, 64), kept.exps)
    d = torch.ones((300, 16), dtype=torch.float16, device="cuda")
    got, want = sp.wgrad(kept, d, km), sp.wgrad(odd, d, km)
    assert _same(got, want)
    assert torch.isinf(got[0, 32]).all() and torch.isfinite(got[0, 33:]).all() and torch.isfinite(got[0, :32]).all()
