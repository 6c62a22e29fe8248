"""Calls on a stream that the caller names, while torch's current stream still has work on memory that was given back to its pool."""
import pytest
import torch

SHAPE = (60_001, 64)


NAMES = ["fwd", "bwd", "pack", "unpack", "relu", "wgrad", "convolution", "its input gradient", "its weight gradient", "add", "map"]


class _Foreign:
    cuda_stream, device_index = 5, 1


def test_a_stream_of_another_device_is_refused():
    from paper_2311_12862_amd import binding
    with pytest.raises(ValueError):
        binding._elsewhere(0, _Foreign(), lambda: None)


def _busy():
    """Some 20 ms of work on the current stream."""
    t = _busy.room = getattr(_busy, "room", None)
    if t is None:
        t = _busy.room = torch.zeros(1 << 28, device="cuda")
    for _ in range(40):
        t.add_(1)


def _tensors():
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dout = (torch.randn(SHAPE, generator=g, device="cuda").half() for _ in range(2))
    return x, dout, 1 + 0.3 * torch.randn(SHAPE[1], generator=g, device="cuda"), 0.3 * torch.randn(SHAPE[1], generator=g, device="cuda")


def _calls():
    """Every call that allocates, by name: f(stream) -> tensors."""
    import paper_2311_12862_amd as sp
    x, dout, w, b = _tensors()
    y, stats = sp.layer_norm_fwd(x, w, b, relu=True)
    kept = sp.q8_pack(y)
    i = torch.arange(SHAPE[0], device="cuda", dtype=torch.int32)
    km = sp.build_kmap(torch.stack([0 * i, i // 256, i % 256, 0 * i], 1).contiguous(), 3, 1)

    k27 = (torch.randn(27, SHAPE[1], SHAPE[1], device="cuda") / 40).half()

    def packed(stream):
        made = sp.q8_pack(x, stream=stream)
        return made.data, made.exps

    return {
        "fwd": lambda s: sp.layer_norm_fwd(x, w, b, relu=True, stream=s),
        "bwd": lambda s: sp.layer_norm_bwd(dout, x, stats, w, gate=kept, residual=True, stream=s),
        "pack": packed,
        "unpack": lambda s: (sp.q8_unpack(kept, torch.float16, stream=s),),
        "relu": lambda s: (sp.ew(sp.EW_RELU_BWD, dout, kept, stream=s),),
        "wgrad": lambda s: (sp.wgrad(kept, dout, km, stream=s),),
        "convolution": lambda s: (sp.fwd(x, k27, km, stream=s),),
        "its input gradient": lambda s: (sp.dgrad(dout, k27, km, stream=s),),
        "its weight gradient": lambda s: (sp.wgrad(x, dout, km, stream=s),),
        "add": lambda s: (sp.ew(sp.EW_ADD, x, dout, stream=s),),
        "map": lambda s: (km.export(stream=s), km.export_mask(stream=s), km.out_coords(stream=s), km.in_coords(stream=s)),
    }


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("named", ["stream", "handle"])
def test_memory_that_the_current_stream_gave_back(name, named):
    """Blocks of every size that the call takes (its workspace's and its results'), given back while the current stream is still to read
    them, keep their values until it has."""
    import paper_2311_12862_amd as sp
    call = _calls()[name]
    want = [t.clone() for t in call(None)]
    sizes = [t.numel() * t.element_size() for t in want]
    if name == "bwd":
        sizes.append(sp.load_library().spconv_layer_norm_bwd_workspace(*SHAPE))
    if name == "pack":                          # (data and exponents are one allocation)
        sizes = [(sizes[0] + 15) // 16 * 16 + sizes[1]]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for turn in range(3):
        given_back = [torch.full((n,), 3, dtype=torch.int8, device="cuda") for n in sizes for _ in range(4)]
        torch.cuda.synchronize()
        _busy()
        late = [t + 1 for t in given_back]      # reads them when the stream gets there
        del given_back
        got = call(side if named == "stream" else side.cuda_stream)
        side.synchronize()
        for a, z in zip(got, want):
            assert torch.equal(a, z)
        torch.cuda.synchronize()
        assert all((t == 4).all() for t in late)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["fwd", "bwd", "unpack", "relu", "convolution", "add"])
def test_results_given_back_while_the_current_stream_reads_them(name):
    import paper_2311_12862_amd as sp
    call = _calls()[name]
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for turn in range(3):
        got = call(side)
        side.synchronize()
        _busy()
        late = [t.clone() for t in got]         # read by the current stream, which is busy,
        del got                                 # and given back at once
        with torch.cuda.stream(side):
            for t in want:
                for _ in range(4):
                    torch.full_like(t, 7)
            sp.layer_norm_fwd(_calls_junk())
        torch.cuda.synchronize()
        assert all(torch.equal(a, z) for a, z in zip(late, want))


def _calls_junk():
    return torch.full(SHAPE, 5.0, dtype=torch.float16, device="cuda")


@pytest.mark.gpu
def test_streams_of_every_kind():
    """The current stream by its object and its handle, the null stream, a side stream as the current one."""
    calls = _calls()
    want = {k: [t.clone() for t in f(None)] for k, f in calls.items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for current in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(current):
            for s in (None, current, current.cuda_stream, 0, torch.cuda.default_stream(), side):
                for k, f in calls.items():
                    got = f(s)
                    torch.cuda.synchronize()
                    assert torch.cuda.current_stream() == current
                    assert all(torch.equal(a, z) for a, z in zip(got, want[k])), k
