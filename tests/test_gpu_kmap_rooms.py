"""Memory that a kmap keeps for its calls: one room, as large as the largest call asked for, and what captured calls replay on."""
import gc

import pytest
import torch

from workloads import generators as gen
from _util import coords_dev

pytestmark = pytest.mark.gpu


class _Blocks:
    """The library's device memory, block by block."""

    def __enter__(self):
        import paper_2311_12862_amd as sp
        self.live = {}

        def alloc(n, stream):
            t = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
            self.live[t.data_ptr()] = t
            return t.data_ptr()

        gc.collect()
        sp.set_allocator(alloc, lambda ptr, stream: self.live.pop(ptr))
        return self

    def __exit__(self, *_):
        import paper_2311_12862_amd as sp
        gc.collect()
        torch.cuda.synchronize()
        sp.set_allocator(None, None)

    def held(self):
        return sum(t.numel() for t in self.live.values())


def _layer(n_in, n_out, ci, co, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n_in, ci, generator=g, device="cuda").to(dtype), torch.randn(n_out, co, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("K,dtype", [(3, torch.float32), (5, torch.float16)])
def test_rooms_of_unpacked_tensors_do_not_add_up(K, dtype):
    import paper_2311_12862_amd as sp
    coords = coords_dev(gen.lidar_scene(51, target_n=3000))
    held = []
    with _Blocks() as blocks:
        for widths in ((64,), (8, 16, 24, 32, 40, 48, 56, 64)):
            km = sp.build_kmap(coords, K, 1)
            for c in widths:
                x, d = _layer(km.n_in, km.n_out, c, 16, dtype, c)
                kept = sp.q8_pack(x)
                got = sp.wgrad(kept, d, km)
                assert torch.equal(got, sp.wgrad(sp.q8_unpack(kept, dtype), d, km))
            torch.cuda.synchronize()
            held.append(blocks.held())
            km.destroy()
            assert not blocks.live
    assert held[1] == held[0]
