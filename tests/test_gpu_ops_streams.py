"""Calls on a stream that is not torch's current one (``stream=``): the same
bits, and memory that no other stream's work shares meanwhile."""
import pytest
import torch

from paper_2608_13966_amd import ops as O

pytestmark = pytest.mark.gpu

DEV = "cuda"
SLEEP = 1 << 21  # of torch's spinning kernel: milliseconds


def rand(*shape, seed=0, dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, device=DEV, generator=g).to(dtype)


def _norm():
    x, res, w = rand(700, 1537, seed=1), rand(700, 1537, seed=2), rand(1537, seed=3)
    return lambda **kw: O.add_rms_norm(x, w, res, quantize=True, **kw)


def _norm_backward():
    x, dy, w = rand(3000, 1537, seed=1), rand(3000, 1537, seed=2), rand(1537, seed=3)
    rstd = x.square().mean(1).add(1e-6).rsqrt()
    return lambda **kw: O.add_rms_norm_backward(dy, x, w, rstd, **kw)


def _distill(what):
    z = rand(6, 140001, seed=1)
    idx, t = torch.topk(z, 32, dim=1)[1], rand(6, 32, seed=2)
    if what == "backward":
        lse = torch.logsumexp(z, 1)
        return lambda **kw: O.distill_topk_backward(z, idx, t, lse, **kw)
    f = O.distill_topk if what == "loss" else O.distill_topk_grad
    return lambda **kw: f(z, idx, t, **kw)


def _linear(m, n=200, k=8192):
    g = torch.Generator(device=DEV).manual_seed(m)
    codes = torch.randint(0, 256, (n * k // 2,), device=DEV, generator=g, dtype=torch.uint8)
    scales, zeros = 0.01 * (1 + rand(n * k // 128, seed=1).abs()), rand(n * k // 128, seed=2)
    w, x = O.PackedWeight(n, k, codes, scales, zeros, bits=4, group=128), rand(m, k, seed=4, dtype=torch.bfloat16)
    return lambda **kw: O.linear_codes(x, w, **kw)


CALLS = {"norm": _norm, "norm_backward": _norm_backward, "distill": lambda: _distill("loss"),
         "distill_backward": lambda: _distill("backward"), "distill_grad": lambda: _distill("grad"),
         "linear_3": lambda: _linear(3), "linear_140": lambda: _linear(140), "linear_1500": lambda: _linear(1500, 4096)}
SHARES = ("norm_backward", "distill", "distill_grad", "linear_3", "linear_140", "linear_1500")  # those with a workspace


def tensors(o, x=None):
    return {k: v for k, v in o.items() if torch.is_tensor(v) and k != "workspace"}


def stream_of_memory(t):
    """The handle of the stream that the caching allocator keeps t's memory for."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_allocates_is_the_streams_own(name):
    call = CALLS[name]()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    before = torch.cuda.current_stream()
    o = call(stream=s.cuda_stream)
    assert torch.cuda.current_stream() == before
    s.synchronize()
    assert (o.get("workspace") is not None) == (name in SHARES)
    for k, t in o.items():
        if torch.is_tensor(t):
            assert stream_of_memory(t) == s.cuda_stream, k
    for k, t in tensors(call(stream=0)).items():  # the default stream by its handle
        assert stream_of_memory(t) == 0, k


@pytest.mark.parametrize("name", CALLS)
def test_dropped_results_are_not_written_over(name):
    """The stream's work comes late; what the call allocated and dropped is the allocator's again before.  The current
    stream allocates and fills as much meanwhile: the outputs that were kept have the right bits all the same."""
    call = CALLS[name]()
    want = tensors(call())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for turn in range(3):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            torch.cuda._sleep(SLEEP)
        o = call(stream=s.cuda_stream)
        space = o.pop("workspace", None)
        size = 0 if space is None else space.numel()
        got = tensors(o)
        del o, space
        junk = [torch.full((max(size, 512),), 255, device=DEV, dtype=torch.uint8) for _ in range(4)]
        s.synchronize()
        for k, t in want.items():
            assert torch.equal(got[k].view(torch.uint8), t.view(torch.uint8)), (k, turn)
        assert all(int(j[0]) == 255 for j in junk)


@pytest.mark.parametrize("name", CALLS)
def test_fresh_memory_is_not_waiting_for_the_current_stream(name):
    """The current stream has writes pending to memory that its program has freed: no output of a call on another
    stream lies there."""
    call = CALLS[name]()
    want = tensors(call())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    freed = [torch.empty_like(t) for t in want.values()]
    torch.cuda._sleep(SLEEP)
    for t in freed:
        t.view(torch.uint8).fill_(255)
    del freed, t
    got = tensors(call(stream=s.cuda_stream))
    torch.cuda.synchronize()
    for k, t in want.items():
        assert torch.equal(got[k].view(torch.uint8), t.view(torch.uint8)), k


def test_no_rows_on_a_stream():
    """The weight gradient of no rows is filled with zeros on the call's stream, not behind the current one's work."""
    x, w = torch.empty(0, 4096, device=DEV), torch.ones(4096, device=DEV)
    rstd = torch.empty(0, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = {"dx": torch.empty(0, 4096, device=DEV), "dw": torch.full((4096,), 7.0, device=DEV)}
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    o = O.add_rms_norm_backward(x, x, w, rstd, out=out, stream=s.cuda_stream)
    with torch.cuda.stream(s):
        host = o["dw"].to("cpu")
    assert (host == 0).all()
    torch.cuda.synchronize()
