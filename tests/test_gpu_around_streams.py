"""GPU: dropout, the norms at a residual joint and log probabilities on a stream of their own
(`stream=`): what they return, and what they take beside it, is of that stream's memory; and two
host threads at once."""

import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
M, N = 300, 1032


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


def calls(pid, layers, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def rand(*shape):
        return torch.randn(shape, generator=g, device=DEV).bfloat16()

    x, o, dh, long = rand(M, N), rand(M, N), rand(M, N), rand(2, 70000)
    w = torch.rand(N, generator=g, device=DEV)
    norm = pid.Norm("rms", w, w)
    block = pid.Block(o, pid.Norm("layer", w, w), w, 0.5, pid.Drop(0.2, 1, 2))
    kept = pid.pointid_norm(layers, x, norm, block, keep=True)
    t = torch.arange(M, dtype=torch.int32, device=DEV)
    lse = pid.pointid_logprobs(layers, x).lse
    torch.cuda.synchronize()
    return {
        "dropout": lambda s: [pid.pointid_dropout(layers, x, pid.Drop(0.5, 3), stream=s)],
        "norm": lambda s: list(pid.pointid_norm(layers, x, norm, block, keep=True, stream=s)),
        "norm_backward": lambda s: list(pid.pointid_norm_backward(layers, dh, kept.total, kept.stats, norm, block, dtotal=x,
                                                                  stream=s)),
        "logprobs": lambda s: list(pid.pointid_logprobs(layers, x, t, entropy=True, top=3, stream=s)),
        "logprobs_long": lambda s: list(pid.pointid_logprobs(layers, long, t[:2], entropy=True, top=30, stream=s)),
        "logprobs_backward": lambda s: [pid.pointid_logprobs_backward(layers, x, lse, t, lse, stream=s)],
    }


NAMES = ["dropout", "norm", "norm_backward", "logprobs", "logprobs_long", "logprobs_backward"]


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
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(s.cuda_stream if raw else s)
    s.synchronize()
    for a, b in zip(got, want):
        assert pool_of(a) == s.cuda_stream and torch.equal(a, b)
    for same in (torch.cuda.current_stream(), 0):
        assert all(torch.equal(a, b) and pool_of(a) == 0 for a, b in zip(call(same), want))
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_the_current_stream_is_busy_with_memory_it_gave_back(pid, layers, name):
    call = calls(pid, layers)[name]
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    held = [torch.empty_like(t) for t in want] + [torch.empty(1 << 22, dtype=torch.uint8, device=DEV)]
    torch.cuda._sleep(100_000_000)                      # some 50 ms
    for t in held:
        t.fill_(5)
    del held, t
    got = call(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_threads_share_the_handle(pid, layers):
    fails = []

    def work(seed):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                mine = calls(pid, layers, seed)
                want = {k: [t.clone() for t in f(None)] for k, f in mine.items()}
                for _ in range(20):
                    for k, f in mine.items():
                        if not all(torch.equal(a, b) for a, b in zip(f(None), want[k])):
                            fails.append((seed, k))
                s.synchronize()
        except Exception as e:                          # noqa: BLE001 - the test reports it
            fails.append((seed, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not fails, fails[:3]


@pytest.mark.parametrize("m, refused", [(400, True), (40, False)])
def test_under_capture_the_handles_scratch_is_refused(pid, layers, m, refused):
    """Rows of one block alone take none: their sums are the sums."""
    x, w = torch.randn((m, 64), device=DEV), torch.ones(64, device=DEV)
    norm = pid.Norm("rms", w)
    got = pid.pointid_norm(layers, x, norm, keep=True)
    want = pid.pointid_norm_backward(layers, x, x, got.stats, norm).dweight
    dw = torch.zeros(64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rc = pid.lib.pointid_norm_backward(layers.raw, 0, m, 64, pid._Matrix(x.data_ptr(), 64), pid._Matrix(x.data_ptr(), 64),
                                           got.stats.data_ptr(), pid._NormOf(1, 1e-5, w.data_ptr(), None), None, None,
                                           pid._NormGrads(None, 0, None, 0, dw.data_ptr()), None, 0,
                                           torch.cuda.current_stream().cuda_stream)
        x.add_(0)
    if refused:
        assert rc == pid.POINTID_EINVAL and "scratch" in pid.pointid_last_error()
        return
    assert rc == pid.POINTID_OK
    for _ in range(3):
        dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, want)
