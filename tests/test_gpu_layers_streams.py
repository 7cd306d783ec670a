"""GPU: calls with a stream of their own (`stream=`): what they return belongs to that stream's
memory, so that no work of the current stream meets it."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def pid():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2009_04509_amd import binding
    return binding


@pytest.fixture(scope="module")
def layers(pid):
    h = pid.pointid_layers_create(0)
    yield h
    h.close()


M, K, N = 300, 264, 520


def calls(pid, layers):
    g = torch.Generator(device=DEV).manual_seed(1)

    def rand(*shape):
        return torch.randn(shape, generator=g, device=DEV).bfloat16()

    x, w, w2, dy, z, u = rand(M, K), rand(K, N), rand(K, N), rand(M, N), rand(M, N), rand(M, N)
    c = pid.pointid_checkpoint_save(z)
    torch.cuda.synchronize()
    return {
        "dense": lambda s: [pid.pointid_dense(layers, x, w, act="silu", stream=s)],
        "dense_backward": lambda s: list(pid.pointid_dense_backward(layers, dy, x, w, z, "silu", stream=s)),
        "gated": lambda s: [pid.pointid_gated(layers, x, w, w2, stream=s)],
        "gated_backward": lambda s: list(pid.pointid_gated_backward(layers, dy, x, w, w2, z, u, need_db=True, stream=s)),
        "checkpoint_save": lambda s: (lambda q: [q.codes, q.exponents])(pid.pointid_checkpoint_save(z, stream=s)),
        "checkpoint_load": lambda s: [pid.pointid_checkpoint_load(c, torch.bfloat16, stream=s)],
    }


NAMES = ["dense", "dense_backward", "gated", "gated_backward", "checkpoint_save", "checkpoint_load"]


def pool_of(t):
    """The stream whose memory a tensor has."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's memory")


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_of_the_calls_stream(pid, layers, name, raw):
    call = calls(pid, layers)[name]
    want = [t.clone() for t in call(None)]              # and leaves the current stream blocks of the same sizes
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(s.cuda_stream if raw else s)
    s.synchronize()
    for a, b in zip(got, want):
        assert pool_of(a) == s.cuda_stream and torch.equal(a, b)
    # the current stream given by name, and the default stream's number
    for same in (torch.cuda.current_stream(), 0):
        assert all(torch.equal(a, b) and pool_of(a) == 0 for a, b in zip(call(same), want))
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_the_current_stream_is_busy_with_memory_it_gave_back(pid, layers, name):
    """The current stream still has to write what it gave back when the call on another stream is
    made: the outputs are not there."""
    call = calls(pid, layers)[name]
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    held = [torch.empty_like(t) for t in want]
    torch.cuda._sleep(100_000_000)                      # some 50 ms
    for t in held:
        t.fill_(5)
    del held, t
    got = call(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
