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


def _calls(km, c, co, dtype):
    """Calls that work in the kmap's own memory: f() -> tensor."""
    import paper_2311_12862_amd as sp
    x, d = _layer(km.n_in, km.n_out, c, co, dtype, c)
    w = torch.randn(km.V, c, co, device="cuda").to(dtype) / 8
    kept = sp.q8_pack(x)
    split, fetch = sp.Config(), sp.Config()
    split.kernel, split.n_split, fetch.kernel = 0 if dtype == torch.float32 else 2, 2, 3
    return {
        "wgrad": lambda: sp.wgrad(x, d, km),
        "wgrad of a checkpoint": lambda: sp.wgrad(kept, d, km),
        "split forward": lambda: sp.fwd(x, w, km, split),
        "fetch on demand": lambda: sp.fwd(x, w, km, fetch),
    }


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("name", ["wgrad", "wgrad of a checkpoint", "split forward", "fetch on demand"])
def test_what_a_captured_call_uses_stays(name, dtype):
    """A wider layer's call after the capture takes no memory from the graph; another kmap and its plans live beside it."""
    import paper_2311_12862_amd as sp
    coords, other = coords_dev(gen.lidar_scene(51, target_n=3000)), coords_dev(gen.lidar_scene(52, target_n=2500))
    with _Blocks() as blocks:
        km = sp.build_kmap(coords, 3, 1)
        call = _calls(km, 32, 16, dtype)[name]
        want = call().clone()
        torch.cuda.synchronize()
        used = set(blocks.live)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for c in (64, 96):
            for f in _calls(km, c, 64, dtype).values():
                f()
        assert used <= set(blocks.live)         # (before anything is replayed)
        beside = sp.build_kmap(other, 3, 1)
        mine = {k: (f, f().clone()) for k, f in _calls(beside, 32, 16, dtype).items() if k != "fetch on demand"}
        tables = beside.export().clone()
        for _ in range(3):
            got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            # (the sums of fetch on demand are atomic: their order is not fixed)
            assert torch.allclose(got, want, rtol=1e-2, atol=1e-2) if name == "fetch on demand" else torch.equal(got, want)
        assert torch.equal(beside.export(), tables)
        assert all(torch.equal(f(), first) for f, first in mine.values())
        torch.cuda.synchronize()
        del graph
        for k in (km, beside):
            k.destroy()
        assert not blocks.live
