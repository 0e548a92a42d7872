"""The reconstruction's calls on a stream that is not torch's current one
(``stream=``): what they allocate belongs to it."""
import pytest
import torch

from paper_2608_13966_amd import quasar as Q

pytestmark = pytest.mark.gpu

DEV = "cuda"


def rand(*shape, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return 0.02 * torch.randn(shape, device=DEV, generator=g)


def stream_of_memory(t):
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


def calls():
    W, g = rand(256, 1024, seed=1), rand(256, 1024, seed=2)
    v, m = g.square(), rand(256, 1024, seed=3)
    amax = W.abs().amax().reshape(1)

    def new(*ts):  # what a call updates in place: there before it, on whatever stream it runs
        made = tuple(t.clone() for t in ts)
        torch.cuda.synchronize()
        return made

    torch.cuda.synchronize()
    return {
        "int": lambda **kw: [Q.reconstruct(W, v, fmt="int", bits=2, group=64, clips=(1.0, 0.9), **kw)],
        "nvfp4": lambda **kw: [Q.reconstruct(W, v, fmt="nvfp4", **kw)],
        "adamw": lambda **kw: [Q.adamw_reconstruct(*new(W, m, v), g, lr=1e-3, bits=4, group=128, **kw)],
        "adamw_nvfp4": lambda **kw: [Q.adamw_reconstruct(*new(W, m, v), g, lr=1e-3, fmt="nvfp4", tensor_amax=amax,
                                                         want_amax_out=True, **kw)],
        "adamw_batch": lambda **kw: Q.adamw_reconstruct_batch([new(W, m, v) + (g,), new(W, m, v) + (g,)], lr=1e-3, **kw),
        "batch": lambda **kw: Q.reconstruct_batch([(W, v, None), (W, v, None)], bits=3, group=128, **kw),
        "batch_nvfp4": lambda **kw: Q.reconstruct_batch([(W, v, None), (W, v, None)], fmt="nvfp4", **kw),
        "absmax": lambda **kw: [{"amax": t} for t in Q.absmax_batch([W, g], **kw)],
    }


@pytest.mark.parametrize("name", ["int", "nvfp4", "adamw", "adamw_nvfp4", "adamw_batch", "batch", "batch_nvfp4", "absmax"])
def test_outputs_belong_to_the_stream(name):
    call = calls()[name]
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(stream=s.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for k, t in a.items():
            if not torch.is_tensor(t):
                continue
            assert stream_of_memory(t) == s.cuda_stream, k
            if k not in ("workspace", "tensor_scale", "amax_out"):
                assert torch.equal(t.view(torch.uint8), b[k].view(torch.uint8)), k
            elif k != "workspace":
                assert torch.equal(t[:1], b[k][:1]), k


def test_absmax_starts_from_zeros_on_its_stream():
    """The zeros that the maximum starts from are there before the kernel, whatever the current stream is at."""
    W = rand(512, 1024, seed=4)
    want = float(W.abs().amax())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(1 << 21)
    out = Q.absmax_batch([W, W], stream=s.cuda_stream)
    with torch.cuda.stream(s):
        assert [float(t[0]) for t in out] == [want, want]
    torch.cuda.synchronize()
    assert [float(t[0]) for t in out] == [want, want]
