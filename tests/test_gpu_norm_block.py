"""A residual block's training step on the library's calls, every activation kept in 8 bits, against the oracle's convolutions and 64-bit
norms: y = ReLU(norm(conv(ReLU(norm(conv(x))))) + x)."""
import numpy as np
import pytest
import torch

from oracle import sparse_conv as oc
from workloads import generators as gen
from _rows import bwd64, fwd64, unpack64
from _util import TOL, coords_dev, make_layer, norm_err

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Block:
    def __init__(self, dtype, c, seed=5):
        import paper_2311_12862_amd as sp
        self.sp, self.dtype, self.c = sp, dtype, c
        coords = gen.lidar_scene(seed, target_n=1500)
        self.ref = oc.build_kmap(coords, 3, 1)
        self.km = sp.build_kmap(coords_dev(coords), 3, 1)
        n = self.ref.n_in
        (self.x32, self.x), (self.w1_32, self.w1), (self.dy32, self.dy) = make_layer(n, n, c, c, 27, dtype, seed)
        _, (self.w2_32, self.w2), _ = make_layer(n, n, c, c, 27, dtype, seed + 50)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g1, self.g2 = (1 + 0.2 * torch.randn(c, generator=g, device="cuda") for _ in range(2))
        self.b1, self.b2 = (0.2 * torch.randn(c, generator=g, device="cuda") for _ in range(2))

    def step(self, x, dy):
        sp, km, (n, c) = self.sp, self.km, x.shape
        kx = sp.q8_pack(x)
        kz1, ka1, kz2, ky = (sp.Checkpoint.empty(n, c) for _ in range(4))
        a1, st1 = sp.layer_norm_fwd(sp.fwd(x, self.w1, km), self.g1, self.b1, EPS, relu=True, keep_x=kz1, keep_y=ka1)
        y, st2 = sp.layer_norm_fwd(sp.fwd(a1, self.w2, km), self.g2, self.b2, EPS, relu=True, residual=x, keep_x=kz2, keep_y=ky)
        dz2, dg2, db2, dres = sp.layer_norm_bwd(dy, kz2, st2, self.g2, gate=ky, residual=True)
        dw2 = sp.wgrad(ka1, dz2, km)
        dz1, dg1, db1, _ = sp.layer_norm_bwd(sp.dgrad(dz2, self.w2, km), kz1, st1, self.g1, gate=ka1)
        dw1 = sp.wgrad(kx, dz1, km)
        dx = sp.ew(sp.EW_ADD, sp.dgrad(dz1, self.w1, km), dres)
        kept = {"x": kx, "z1": kz1, "a1": ka1, "z2": kz2, "y": ky, "st1": st1, "st2": st2}
        return {"y": y, "dx": dx, "dw1": dw1, "dw2": dw2, "dg1": dg1, "db1": db1, "dg2": dg2, "db2": db2}, kept


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype,c", [("f32", 32), ("f32", 20), ("f16", 64), ("bf16", 96), ("f16", 40)])
def test_block(dtype, c):
    b = Block(dtype, c)
    out, kept = b.step(b.x, b.dy)
    M, n = b.ref.M, b.ref.n_in
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).double()  # noqa: E731
    p = {k: getattr(b, k).cpu() for k in ("g1", "b1", "g2", "b2")}
    # forward
    a1 = fwd64(dev(oc.forward(b.x32, b.w1_32, M)), p["g1"], p["b1"], EPS, True, None)[0]
    y = fwd64(dev(oc.forward(a1.numpy(), b.w2_32, M)), p["g2"], p["b2"], EPS, True, dev(b.x32))[0]
    assert norm_err(out["y"], y.numpy()) <= TOL[dtype]
    # backward at the values that were kept (which is what the step computes), in 64 bits from dy on
    v = {k: unpack64(t.data.cpu(), t.exps.cpu()) for k, t in kept.items() if not k.startswith("st")}
    want, _ = bwd64(dev(b.dy32), v["z2"], kept["st2"].cpu(), p["g2"], v["y"] > 0)
    dz2, ref = want[0].numpy(), {"dg2": want[1], "db2": want[2]}
    ref["dw2"] = oc.wgrad(v["a1"].numpy(), dz2, M)
    want1, _ = bwd64(dev(oc.dgrad(dz2, b.w2_32, M, n)), v["z1"], kept["st1"].cpu(), p["g1"], v["a1"] > 0)
    dz1 = want1[0].numpy()
    ref |= {"dg1": want1[1], "db1": want1[2], "dw1": oc.wgrad(v["x"].numpy(), dz1, M), "dx": oc.dgrad(dz1, b.w1_32, M, n) + want[3].numpy()}
    for name, r in ref.items():
        assert norm_err(out[name], _np(r) if torch.is_tensor(r) else r) <= TOL[dtype], name


def test_block_replays_in_a_hip_graph():
    """The whole step captured, replayed on new inputs with eager steps of the same block in between."""
    b = Block("f16", 64)
    x, dy = b.x.clone(), b.dy.clone()
    b.step(x, dy)                                    # plans, pair list and scratch exist from here on
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs, _ = b.step(x, dy)
    for replay in range(4):
        x.copy_(b.x.roll(replay, 0))
        dy.copy_(b.dy.roll(2 * replay, 1))
        want = {k: t.clone() for k, t in b.step(x, dy)[0].items()}
        graph.replay()
        torch.cuda.synchronize()
        for k, t in outs.items():
            assert torch.equal(t, want[k]), (replay, k)
